// sq_sparse_attn_decode_q8: decode attention over e4m3 keys and values, kept ranges of the fixed context and the pages of the
// user cache, one softmax over both.
//
// A row is a (sequence, K/V head) with its g query heads (one kept set) or a single query head.  Its keys, laid end to end --
// the kept keys of the fixed context, then the user's -- are cut into tiles of 32; the tiles of all rows, laid end to end, are cut
// into equal shares, one per workgroup, so rows that keep more get more of the chip.  What bounds it is the 256 bytes of a key and
// its value, read once per row.
//
// A wave lists 64 keys at a time, a step before it reads them, by itself: no barrier stands between two tiles, and two workgroups a CU
// hide the reads (Q8_GRID; the registers and LDS of three would fit where offsets have 32 bits, which was not measured).  Two tiles on
// their way instead of one are slower (32 heads 16 -> 18 us).  Measured, kernel and merge:
//   8 sequences x 8 heads of 4 queries with one set, 128K keys of which 1/16, up to 16K user keys (318 MB): 62 + 5 us, 4.8 TB/s
//   32 heads, 32K keys of which 1/8, 512 user keys (38 MB):           13 + 4 us: a chain of reads (the row's numbers, its ranges, the
//                                                                     scales, keys, values), a tile or two a wave, and a second launch
//   4 heads, 4096 keys of which 1/4, 128 user keys (1.2 MB):          7 + 3 us, as long as the calling thread takes for two launches
#include "sq_decode_q8.hpp"

namespace sq {

namespace {

constexpr int SENTINEL = INT32_MIN;
constexpr int GROUP = 64;                    // ranges that a wave holds at a time
constexpr int MAX_GROUPS = SELECT_MAX_C / GROUP;

struct RowTiles {
    int nf, nu, tf, total;                   // fixed and user keys, tiles of fixed keys, all tiles (at least one)
};

__device__ __forceinline__ RowTiles tiles_of(int nf, int nu)
{
    const int tf = (nf + QT - 1) / QT;
    return RowTiles{nf, nu, tf, max(1, tf + (nu + QT - 1) / QT)};
}
// A row's numbers, read side by side without a branch (of what is not there, some number that is not used).
struct RowKeys {
    int nf, nu;
};
__device__ __forceinline__ RowKeys read_row(const DecodeQ8Args &a, const Row &w)
{
    const int32_t *nf = a.ranges ? a.n_keys + w.r : a.seq_len, *nu = a.seq_len ? a.seq_len + w.b : a.n_keys;
    return RowKeys{*nf, *nu};
}
__device__ __forceinline__ RowTiles row_tiles(const DecodeQ8Args &a, const RowKeys &n)
{
    return tiles_of(a.ranges ? min(max(n.nf, 0), a.L) : 0, a.seq_len ? min(max(n.nu, 0), a.max_pages << a.p_log) : 0);
}
__device__ __forceinline__ RowTiles row_tiles(const DecodeQ8Args &a, int i) { return row_tiles(a, read_row(a, dealt_row(a, i))); }

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

}  // namespace

template <bool WIDE>
__global__ __launch_bounds__(256, 2) void decode_q8_kernel(DecodeQ8Args a)
{
    typedef decltype(KeyList<WIDE>::at[0] + 0) offset_t;
    __shared__ __align__(16) WaveOut s_out;
    __shared__ __align__(16) KeyList<WIDE> s_list[4][2];
    __shared__ __align__(16) offset_t s_none[QT];           // where a wave reads ahead behind its last tile: the first row, a line or two
    __shared__ int s_delta[4][64];
    __shared__ int s_group[MAX_GROUPS];
    __shared__ int s_w[4], s_found[4];
    __shared__ float s_ml[2][4][16];

    const int wave = uniform(threadIdx.x >> 6);

    const int tid = threadIdx.x;
    if (tid < QT) s_none[tid] = 0;
    __syncthreads();
    // This workgroup's share: tiles [t0, t1), counted from row ri's first less row_start; share0 + t / per is who has tile t.
    int share, share0, per, t0, t1, ri, row_start;
    RowTiles rt;
    if (a.splits > 0) {
        // Few keys: a row's tiles are divided among workgroups of its own, without a look at the other rows.
        ri = blockIdx.x / a.splits;
        rt = row_tiles(a, ri);
        rt = tiles_of(uniform(rt.nf), uniform(rt.nu));
        share0 = ri * a.splits;
        share = blockIdx.x;
        per = max(4, (rt.total + a.splits - 1) / a.splits);
        row_start = 0;
        t0 = (share - share0) * per;
        t1 = min(rt.total, t0 + per);
        if (t0 >= t1) return;
    } else {
        // Workgroups go round the 8 XCDs: each XCD takes consecutive shares.
        const int R = a.B * a.H * a.per;
        auto divide = [&](int all) {                        // false: no share for this workgroup
            const int shares = min((int)gridDim.x, (all + 3) / 4), per_xcd = (shares + 7) / 8;      // (at least a tile for each wave)
            per = (all + shares - 1) / shares;
            share0 = 0;
            share = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
            if ((int)(blockIdx.x >> 3) >= per_xcd || (long long)share * per >= all) return false;
            t0 = share * per;
            t1 = min(all, t0 + per);
            return true;
        };
        int nf, nu;
        if (R <= Q8_WAVE_ROWS) {
            // every wave for itself, four rows a lane
            const int lane = tid & 63;
            Row rows[4];
            RowKeys n[4];
            RowTiles mine[4];
            int sum = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) rows[k] = dealt_row(a, min(4 * lane + k, R - 1));
#pragma unroll
            for (int k = 0; k < 4; ++k) n[k] = read_row(a, rows[k]);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                mine[k] = row_tiles(a, n[k]);
                if (4 * lane + k >= R) mine[k].total = 0;
                sum += mine[k].total;
            }
            const int inc = wave_inclusive_scan(sum, lane);
            if (!divide(__builtin_amdgcn_readlane(inc, 63))) return;
            int before = inc - sum, at = 0;
            const unsigned long long here = __ballot(before <= t0 && t0 < inc);
            const int owner = __ffsll((long long)here) - 1;
            nf = mine[0].nf;
            nu = mine[0].nu;
#pragma unroll
            for (int k = 0; k < 3; ++k)
                if (at == k && t0 >= before + mine[k].total) {
                    before += mine[k].total;
                    at = k + 1;
                    nf = mine[k + 1].nf;
                    nu = mine[k + 1].nu;
                }
            ri = __builtin_amdgcn_readlane(4 * lane + at, owner);
            row_start = __builtin_amdgcn_readlane(before, owner);
            nf = __builtin_amdgcn_readlane(nf, owner);
            nu = __builtin_amdgcn_readlane(nu, owner);
        } else {
            const int each = (R + 255) / 256, i_lo = min(R, tid * each), i_hi = min(R, i_lo + each);
            int mine = 0, all;
            for (int i = i_lo; i < i_hi; ++i) mine += row_tiles(a, i).total;
            int before = block_exclusive(mine, tid, s_w, all);
            if (!divide(all)) return;
            if (before <= t0 && t0 < before + mine) {
                int i = i_lo;
                for (;; ++i) {
                    rt = row_tiles(a, i);
                    if (t0 < before + rt.total) break;
                    before += rt.total;
                }
                s_found[0] = i;
                s_found[1] = before;
                s_found[2] = rt.nf;
                s_found[3] = rt.nu;
            }
            __syncthreads();
            ri = s_found[0];
            row_start = s_found[1];
            nf = s_found[2];
            nu = s_found[3];
        }
        // (a row's numbers are the same in every lane: known to be, they take scalar registers, and addresses a scalar base)
        ri = uniform(ri);
        row_start = uniform(row_start);
        rt = tiles_of(uniform(nf), uniform(nu));
    }

    for (;;) {
        const int lane = thread_here() & 63, c16 = lane & 15, g4 = lane >> 4;
        const Row row = dealt_row(a, ri);
        const int r = row.r, h = row.h, b = row.b;
        const int lo = max(t0 - row_start, 0), hi = min(t1 - row_start, rt.total);
        Attending st;
        begin(st);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const h8 zero = {};
            st.q[s] = c16 < a.g ? *reinterpret_cast<const h8 *>(a.q + ((size_t)r * a.g + c16) * D + 32 * g4 + 8 * s) : zero;
        }

        // The row's ranges in groups of 64: how many keys lie before each group, for a wave to find its first.
        const global<i2v> rg = uniform(reinterpret_cast<const i2v *>(a.ranges) + (size_t)r * a.C);
        const bool has_fixed = lo < rt.tf;
        // Up to four of them every wave has in registers, read beside the number of ranges and not behind it; more are summed by turns.
        auto range_of = [&](int gi) { return rg[min(gi * GROUP + lane, a.C - 1)]; };   // as it stands in memory: see in_bounds
        i2v near[4] = {};
        if (has_fixed) {
#pragma unroll
            for (int k = 0; k < 4; ++k) near[k] = range_of(k);
        }
        const int nr = uniform(has_fixed ? min(max(a.n_ranges[r], 0), a.C) : 0), groups = (nr + GROUP - 1) / GROUP;
        auto in_bounds = [&](i2v e, int gi) {               // a lane's range of a group; (0, 0) behind the last
            const bool ok = gi * GROUP + lane < nr;
            return i2v{min(max(e.x, -MAX_L), MAX_L), ok ? min(max(e.y, 0), a.L) : 0};
        };
        if (groups > 4) {
            for (int gi = wave; gi < groups; gi += 4) {
                // (counts that sum to more than a row can have are cut, far from overflow)
                const int n = min(wave_sum_i(in_bounds(range_of(gi), gi).y), MAX_L);
                if (lane == 0) s_group[gi] = n;
            }
            __syncthreads();
        }

        // This wave's quarter of the tiles: fixed keys, then the user's, 64 keys listed at a time and a step ahead.
        const int w0 = lo + (int)((long long)(hi - lo) * wave / 4), w1 = lo + (int)((long long)(hi - lo) * (wave + 1) / 4);
        int phase = 0;
#pragma clang loop unroll(disable)
        for (; phase < 2; ++phase) {
            asm volatile("" : "+s"(phase));                 // (one copy of the loop below for both)
            const bool fixed = phase == 0;
            const int f0 = fixed ? w0 : max(w0, rt.tf) - rt.tf;          // first tile of the phase, and how many
            const int tiles = (fixed ? min(w1, rt.tf) : w1 - rt.tf) - f0;
            // (the one tile of a row without keys reads nothing: where there is no cache there is no first row either)
            if (tiles <= 0 || (!fixed && rt.nu == 0)) continue;
            const size_t head = fixed ? (size_t)h * a.L * D : 0;
            const global<uint8_t> Kb = uniform((fixed ? a.K8 : a.cK) + head), Vb = uniform((fixed ? a.V8 : a.cV) + head);
            const global<float> kscale = uniform(fixed ? a.ks : a.cks), vscale = uniform(fixed ? a.vs : a.cvs);
            const global<int32_t> pages = uniform(a.page_table + (size_t)b * a.max_pages);
            int p = f0 * QT;                                // the next position to list
            int end;                                        // where the row's keys end
            // ranges in hand: group gi, its lanes' first positions, where it ends; the group behind it is on its way
            int gi = 0, first = 0, ends = 0;
            i2v e = {0, 0}, e_next = {0, 0};                 // user: e.x is the page of position p + lane, read ahead
            if (fixed) {
                int start = 0, total = 0;                   // keys before group gi, keys of all groups
                if (groups <= 4) {
                    e = in_bounds(near[0], 0);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        total += wave_sum_i(in_bounds(near[k], k).y);
                        if (k + 1 < groups && total <= p) {
                            gi = k + 1;
                            start = total;
                            e = in_bounds(near[k < 3 ? k + 1 : 3], k + 1);
                        }
                    }
                    total = uniform(total);
                } else {
                    int sum[MAX_GROUPS / 64], at = 0;
#pragma unroll
                    for (int i = 0; i < MAX_GROUPS / 64; ++i) {
                        sum[i] = 4 * lane + i < groups ? s_group[4 * lane + i] : 0;
                        at += sum[i];
                    }
                    const int inc = wave_inclusive_scan(at, lane);
                    total = __builtin_amdgcn_readlane(inc, 63);
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
                end = min(rt.nf, total);
                e_next = range_of(gi + 1);
                const int c = wave_inclusive_scan(e.y, lane);
                first = start + c - e.y;
                ends = uniform(start + __builtin_amdgcn_readlane(c, 63));
            } else {
                end = rt.nu;
                e.x = -1;
                if (end > 0) e.x = pages[min(p + lane, end - 1) >> a.p_log];
            }

            float ks = 0.0f, vs = 0.0f;
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
                    if (end > 0) e.x = pages[min(t + 64, end - 1) >> a.p_log];
                }
                ks = vs = 0.0f;
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
                s_list[wave][buf].ks[lane] = ks * a.scale;
                s_list[wave][buf].vs[lane] = vs;
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
                const float *kf = s_list[wave][buf].ks + slot + 4 * g4, *vf = s_list[wave][buf].vs + slot + 4 * g4;
                fold_tile(
                    st, k, v, kf, vf, [&]() { load_k(t + 1); },  // (as soon as the scores have used this tile's)
                    [&](float(&x)[8], uint32_t(&w)[2][8]) {
                        const uint32_t keys = (uint32_t)(seen >> slot);
                        if (keys != 0xffffffffu) hide_empty(x, w, keys >> (4 * g4));
                    });
                load_v(t + 1);
                if (even && t + 2 < tiles) list_scales(buf ^ 1);
            }
        }
        // The four waves' results of the row.
        hand_over(st, a.g, wave, s_out, s_ml);
        __syncthreads();
        const int tid = thread_here();
        const bool whole = lo == 0 && hi == rt.total;
        const int slot = share + ri;
        for (int i = tid; i < a.g * D; i += 256) {
            const int qi = i >> 7, d = i & 127;
            const Joined x = join(s_out, s_ml, qi, d);
            if (whole) store_result(a, (size_t)r * a.g + qi, d, x.m, x.l, x.o);
            else store_partial(a.part + ((size_t)slot * a.g + qi) * PART_STRIDE, d, x);
        }
        if (tid == 0 && lo == 0) {
            const int last = share0 + (row_start + rt.total - 1) / per;
            a.info[r] = int2{slot, whole ? 0 : last - share + 1};
        }
        __syncthreads();
        row_start += rt.total;
        if (row_start >= t1) break;
        ++ri;
        const RowTiles next = row_tiles(a, ri);
        rt = tiles_of(uniform(next.nf), uniform(next.nu));
    }
}

// Rows that several workgroups took: one workgroup per row and query.  Eight groups of 32 lanes fold every eighth partial result,
// a lane four dimensions, and are folded in LDS.
__global__ __launch_bounds__(256) void decode_q8_merge_kernel(DecodeQ8Args a)
{
    const int r = blockIdx.x / a.g, qi = blockIdx.x - r * a.g, tid = threadIdx.x, grp = tid >> 5, quad = tid & 31;
    __shared__ float s_m[8], s_l[8];
    __shared__ __align__(16) float s_o[8][D];
    // where the query's partial results are: the first, how many, how far apart
    size_t first;
    int n, step;
    if (a.groups > 0) {
        const int i = r % a.per, bh = r / a.per, h = bh % a.H, in_head = bh / a.H * a.per + i;
        const int grp = in_head / a.rows_per_group, column = (in_head - grp * a.rows_per_group) * a.g + qi;
        first = ((size_t)h * a.groups + grp) * a.parts * 16 + column;
        n = a.parts;
        step = 16;
    } else {
        const int2 info = a.info[r];
        if (info.y == 0) return;
        first = (size_t)info.x * a.g + qi;
        n = info.y;
        step = a.g;
    }
    float M = SQ_NEG_INF, ls = 0.0f;
    f4 os = {0.f, 0.f, 0.f, 0.f};
    auto part = [&](int i) { return a.part + (first + (size_t)i * step) * PART_STRIDE; };
    auto fold = [&](float pm, float pl, f4 po) {
        const float mn = fmaxf(M, pm), mu = mn == SQ_NEG_INF ? 0.0f : mn;
        const float fa = exp2f(M - mu), fb = exp2f(pm - mu);
        ls = ls * fa + pl * fb;
        os = os * fa + po * fb;
        M = mn;
    };
    int i = grp;
    for (; i + 8 < n; i += 16) {
        const float *p = part(i), *q = part(i + 8);
        const float2 a0 = *reinterpret_cast<const float2 *>(p), a1 = *reinterpret_cast<const float2 *>(q);
        const f4 o0 = *reinterpret_cast<const f4 *>(p + 4 + 4 * quad), o1 = *reinterpret_cast<const f4 *>(q + 4 + 4 * quad);
        fold(a0.x, a0.y, o0);
        fold(a1.x, a1.y, o1);
    }
    if (i < n) {
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

hipError_t launch_decode_q8(const DecodeQ8Args &args, hipStream_t s)
{
    DecodeQ8Args a = args;
    const bool wide = ((size_t)a.n_pages * a.H << a.p_log) * D > (1ull << 32);
    hipEvent_t ev0 = nullptr, ev1 = nullptr;
    const bool timed = profile_pair(&ev0, &ev1);
    const Q8Groups shared = a.ranges ? q8_groups(a.B, a.H, a.per, a.g, a.L) : Q8Groups{0, 0, 0};
    a.groups = shared.groups;
    if (shared.groups > 0) {
        a.rows_per_group = shared.rows;
        a.parts = shared.parts;
        launch_decode_q8_shared(a, wide, timed ? ev0 : nullptr, ev1, s);
    } else {
        const long long rows = (long long)a.B * a.H * a.per, most = (a.ranges ? a.L : 0) + (a.seq_len ? a.max_pages << a.p_log : 0);
        a.splits = q8_splits(rows, most);
        const int grid = a.splits ? (int)rows * a.splits : Q8_GRID;
        auto *kernel = wide ? decode_q8_kernel<true> : decode_q8_kernel<false>;
        if (timed) hipExtLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, s, ev0, ev1, 0, a);
        else hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, s, a);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(decode_q8_merge_kernel, dim3((unsigned)(a.B * a.H * a.per * a.g)), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace sq
