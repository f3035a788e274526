// sq_sparse_attn_decode_q8 where eight rows or more read one head of the fixed context: sequences that share it, query heads of a K/V
// head that select on their own.
//
// The rows of a head are taken in groups that fill the 16 columns of a tile.  A workgroup has a group and every S-th window of 256 keys
// of its head: it marks what each row keeps there (a bit per key and row), lists the keys that some row keeps, and folds each of them
// once for all rows, the scores of rows that do not keep it hidden.  So a key that several rows keep is read once, not once per row;
// what bounds it is the 256 bytes of a key and its value over the union of the rows' sets.  The rows' own user keys follow in the same
// way, hidden from the other rows, and divided among the S workgroups of the group, each of which leaves one partial result per query.
// 16 sequences over 32 heads of 32K keys that keep 1/8 each, up to 256 user keys (264 MB with the union; the rows by themselves 550 MB):
// 60 + 5 us for the kernel and the merge, 4.4 TB/s, where the rows by themselves take 89.  Marking, listing and folding take the vector
// units 25 us of that (15.2 million vector instructions of 4 cycles over 1024 SIMDs), at two workgroups a CU (Q8_SHARED_GRID; three would
// fit where offsets have 32 bits, which was not measured).  Each workgroup reads the ranges of all its rows to find its own windows,
// whatever the rows keep: that is most of the time where they keep little.
//
// A NaN among the values of a key that is hidden from a row would still reach it, as zero times NaN.  A workgroup that ends with a NaN
// therefore takes its rows again, one by one, with that row's keys only.
#include "sq_decode_q8.hpp"

namespace sq {

namespace {

constexpr int WINDOW = Q8_WINDOW;            // keys of a window, in words of 64 bits
constexpr int WINDOW_WORDS = WINDOW / 64;
constexpr int BATCH_WORDS = 64;              // words that are held at a time
constexpr int BATCH = BATCH_WORDS / WINDOW_WORDS;

}  // namespace

template <bool WIDE, bool STREAM>
__global__ __launch_bounds__(256, 2) void decode_q8_shared_kernel(DecodeQ8Args a)
{
    typedef decltype(KeyList<WIDE>::at[0] + 0) offset_t;
    __shared__ __align__(16) WaveOut s_out;
    __shared__ __align__(16) KeyList<WIDE> s_list[4][2];
    __shared__ __align__(16) offset_t s_none[QT];           // where a wave reads ahead behind its last tile: the first row
    __shared__ __align__(16) unsigned short s_rows[4][2][64];   // per listed key: the rows that see it
    __shared__ int s_key[4][128];                           // keys of the union on their way into a list, and their rows
    __shared__ unsigned short s_key_rows[4][128];
    __shared__ __align__(8) uint32_t s_bits[16][2 * BATCH_WORDS];
    __shared__ float s_ml[2][4][16];

    const int wave = uniform(threadIdx.x >> 6);
    if (threadIdx.x < QT) s_none[threadIdx.x] = 0;
    // units (head, group of rows, s of S), consecutive ones on the same XCD
    const int S = a.parts, units = a.H * a.groups * S, per_xcd = (units + 7) / 8;
    const int unit = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per_xcd || unit >= units) return;
    const int hg = unit / S, s = unit - hg * S, h = hg / a.groups, grp = hg - h * a.groups;
    const int in_head = a.B * a.per, first_row = h * in_head + grp * a.rows_per_group;
    const int nj = min(a.rows_per_group, in_head - grp * a.rows_per_group), columns = nj * a.g;
    const int windows = (a.L + WINDOW - 1) / WINDOW, mine = (windows - s + S - 1) / S, batches = a.ranges ? (mine + BATCH - 1) / BATCH : 0;
    const global<uint8_t> Kf = uniform(a.K8 + (size_t)h * a.L * D), Vf = uniform(a.V8 + (size_t)h * a.L * D);

    // only < 0: all rows; otherwise that row alone, after a NaN
    for (int only = -1; only < nj; ++only) {
        const int lane = thread_here() & 63, c16 = lane & 15, g4 = lane >> 4;
        Attending st;
        begin(st);
        const int my_row = c16 / a.g;                       // this lane's column: row of the group, query of the row
        const Row w = dealt_row(a, first_row + min(my_row, nj - 1));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const h8 zero = {};
            st.q[i] = c16 < columns ? *reinterpret_cast<const h8 *>(a.q + ((size_t)w.r * a.g + c16 % a.g) * D + 32 * g4 + 8 * i) : zero;
        }
        const uint32_t bit = 1u << my_row;
        // user keys of row c16 (not of column c16): how many, and the 64-key chunks of it and of those before it
        const Row u = dealt_row(a, first_row + min(c16, nj - 1));
        int held = 0;
        if (a.seq_len && c16 < nj) held = min(max(a.seq_len[u.b], 0), a.max_pages << a.p_log);
        int chunks_to = (held + 63) >> 6;
        const int chunks_of = chunks_to;
        chunks_to += dpp_i0<0x111>(chunks_to);              // inclusive sums over the 16 lanes
        chunks_to += dpp_i0<0x112>(chunks_to);
        chunks_to += dpp_i0<0x114>(chunks_to);
        chunks_to += dpp_i0<0x118>(chunks_to);
        const int chunks = __builtin_amdgcn_readlane(chunks_to, 15), my_chunk = s * 4 + wave;

        int batch = 0;
#pragma clang loop unroll(disable)
        for (; batch <= batches; ++batch) {
            asm volatile("" : "+s"(batch));                 // (one copy of the loop below for both kinds of keys)
            const bool fixed = batch < batches;
            int tiles;
            if (fixed) {
                __syncthreads();
                for (int i = threadIdx.x; i < 16 * 2 * BATCH_WORDS; i += 256) s_bits[0][i] = 0u;
                __syncthreads();
                for (int j = wave; j < nj; j += 4) {
                    if (only >= 0 && j != only) continue;
                    const int r = uniform(dealt_row(a, first_row + j).r);
                    const int nr = uniform(min(max(a.n_ranges[r], 0), a.C));
                    const global<i2v> rg = uniform(reinterpret_cast<const i2v *>(a.ranges) + (size_t)r * a.C);
                    for (int i0 = 0; i0 < nr; i0 += 256) {
                        i2v e[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) e[k] = rg[min(i0 + 64 * k + lane, a.C - 1)];
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            if (i0 + 64 * k + lane >= nr) continue;
                            const int x = min(max(e[k].x, -MAX_L), MAX_L), y = min(max(e[k].y, 0), a.L);
                            const int lo = min(max(x, 0), a.L), hi = min(max(x + y, lo), a.L);
                            // this workgroup's windows that the range touches, from the batch's first on
                            int at = max((lo / WINDOW - s + S - 1) / S, batch * BATCH);
                            int win = at * S + s;
                            at -= batch * BATCH;
                            for (; win * WINDOW < hi && at < BATCH; win += S, ++at) {
                                const int from = max(lo - win * WINDOW, 0), to = min(hi - win * WINDOW, WINDOW);
                                uint32_t *row = &s_bits[j][at * (WINDOW / 32)];
                                for (int b = from >> 5; b <= (to - 1) >> 5 && from < to; ++b)
                                    atomicOr(&row[b], (~0u << max(from - 32 * b, 0)) & (~0u >> max(32 * b + 32 - to, 0)));
                            }
                        }
                    }
                }
                __syncthreads();
            } else {
                tiles = my_chunk < chunks ? 2 * ((chunks - my_chunk + 4 * S - 1) / (4 * S)) : 0;
            }
            // Word w of the batch: 64 consecutive keys; the union of its rows' bits, the same in every lane.  A wave has words wave, wave + 4, ..
            auto word_of = [&](int i, uint32_t &lo, uint32_t &hi) {   // this lane's row's bits of the wave's i-th word
                const uint32_t *p = &s_bits[c16][2 * (wave + 4 * i)];
                lo = p[0];
                hi = p[1];
            };
            auto any_row = [&](uint32_t v) {
                v |= (uint32_t)dpp_i0<0x128>((int)v);
                v |= (uint32_t)dpp_i0<0x124>((int)v);
                v |= (uint32_t)dpp_i0<0x122>((int)v);
                v |= (uint32_t)dpp_i0<0x121>((int)v);
                return v;
            };
            if (fixed) {
                int n = 0;
                for (int i = 0; i < BATCH_WORDS / 16; ++i) {
                    uint32_t lo, hi;
                    word_of(4 * i + g4, lo, hi);            // (four words at a time)
                    n += __popc(any_row(lo)) + __popc(any_row(hi));
                }
                n = __builtin_amdgcn_readlane(n, 0) + __builtin_amdgcn_readlane(n, 16) + __builtin_amdgcn_readlane(n, 32) + __builtin_amdgcn_readlane(n, 48);
                tiles = (n + QT - 1) / QT;
            }
            tiles = uniform(tiles);
            if (tiles <= 0) continue;
            const global<uint8_t> Kb = fixed ? Kf : uniform(a.cK), Vb = fixed ? Vf : uniform(a.cV);
            const global<float> kscale = uniform(fixed ? a.ks : a.cks), vscale = uniform(fixed ? a.vs : a.cvs);

            int word = 0, have = 0;                         // fixed: the next word, keys in s_key
            int chunk = my_chunk;                           // user: the next chunk of 64 keys, the page of its keys read ahead
            auto locate = [&](int c, int &j, int &t) {      // row of a chunk, its lane's token
                j = min(__popcll(__ballot(lane < 16 && chunks_to <= c)), 15);
                t = (c - __builtin_amdgcn_readlane(chunks_to - chunks_of, j)) * 64 + lane;
            };
            auto page_of = [&](int c) {
                int j, t;
                locate(c, j, t);
                const int end = __builtin_amdgcn_readlane(held, j), seq = __builtin_amdgcn_readlane(u.b, j);
                return c < chunks ? a.page_table[(size_t)seq * a.max_pages + (min(t, end - 1) >> a.p_log)] : -1;
            };
            int page = fixed ? -1 : page_of(chunk);
            float ks = 0.0f, vs = 0.0f;
            unsigned long long seen = 0ull, seen_next = 0ull;
            auto list = [&](int buf) {
                offset_t at = 0;
                int sc = 0;
                uint32_t rows = 0;
                if (fixed) {
                    while (have < 64 && word < BATCH_WORDS / 4) {
                        uint32_t lo, hi;
                        word_of(word, lo, hi);
                        const uint32_t ulo = __builtin_amdgcn_readlane((int)any_row(lo), 0), uhi = __builtin_amdgcn_readlane((int)any_row(hi), 0);
                        const unsigned long long some = (unsigned long long)uhi << 32 | ulo;
                        const int at_word = wave + 4 * word;
                        ++word;
                        if (some == 0ull) continue;
                        uint32_t m = 0;
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            const uint32_t wl = __builtin_amdgcn_readlane((int)lo, j), wh = __builtin_amdgcn_readlane((int)hi, j);
                            m |= __builtin_amdgcn_inverse_ballot_w64((unsigned long long)wh << 32 | wl) ? 1u << j : 0u;
                        }
                        if (m != 0u) {
                            const int to = have + __popcll(some & ((1ull << lane) - 1ull));
                            const int win = (batch * BATCH + at_word / WINDOW_WORDS) * S + s;
                            s_key[wave][to] = win * WINDOW + at_word % WINDOW_WORDS * 64 + lane;
                            s_key_rows[wave][to] = (unsigned short)m;
                        }
                        have = uniform(have + __popcll(some));
                    }
                    wave_lds_sync();
                    if (lane < have) {
                        const int key = s_key[wave][lane];
                        rows = s_key_rows[wave][lane];
                        at = (offset_t)key * D;
                        sc = h * a.sblocks + (key >> 6);
                    }
                    const int rest = s_key[wave][64 + lane];
                    const unsigned short rest_rows = s_key_rows[wave][64 + lane];
                    wave_lds_sync();
                    if (64 + lane < have) {
                        s_key[wave][lane] = rest;
                        s_key_rows[wave][lane] = rest_rows;
                    }
                    have = max(have - 64, 0);
                } else {
                    int j, t;
                    locate(chunk, j, t);
                    // (a row taken again alone has the chunks that it had)
                    if ((only < 0 || only == j) && t < __builtin_amdgcn_readlane(held, j) && page >= 0 && page < a.n_pages) {
                        sc = page * a.H + h;
                        at = (((offset_t)sc << a.p_log) + (t & ((1 << a.p_log) - 1))) * D;
                        rows = 1u << j;
                    }
                    chunk += 4 * S;
                    page = page_of(chunk);
                }
                ks = vs = 0.0f;
                if (rows != 0u) {
                    ks = kscale[sc];
                    vs = vscale[sc];
                }
                s_list[wave][buf].at[lane] = at;
                s_rows[wave][buf][lane] = (unsigned short)rows;
                seen_next = __ballot(rows != 0u);
                wave_lds_sync();
            };
            auto list_scales = [&](int buf) {
                s_list[wave][buf].ks[lane] = ks * a.scale;
                s_list[wave][buf].vs[lane] = vs;
                wave_lds_sync();
            };
            u4v k[2][2];
            u2v v[8];
            auto load_k = [&](int t) {
                const auto *at = t < tiles ? s_list[wave][(t >> 1) & 1].at + (t & 1) * QT : s_none;
                const offset_t k0 = at[c16] + 32 * g4, k1 = at[16 + c16] + 32 * g4;
                k[0][0] = load_once<STREAM>(reinterpret_cast<global<u4v>>(Kb + k0));
                k[0][1] = load_once<STREAM>(reinterpret_cast<global<u4v>>(Kb + k0 + 16));
                k[1][0] = load_once<STREAM>(reinterpret_cast<global<u4v>>(Kb + k1));
                k[1][1] = load_once<STREAM>(reinterpret_cast<global<u4v>>(Kb + k1 + 16));
            };
            auto load_v = [&](int t) {
                const auto *at = (t < tiles ? s_list[wave][(t >> 1) & 1].at + (t & 1) * QT : s_none) + 4 * g4;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    v[i] = load_once<STREAM>(reinterpret_cast<global<u2v>>(Vb + (offset_t)(at[(i < 4 ? 0 : 12) + i] + 8 * c16)));
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
                const u2v r0 = *reinterpret_cast<const u2v *>(&s_rows[wave][buf][slot + 4 * g4]);
                const u2v r1 = *reinterpret_cast<const u2v *>(&s_rows[wave][buf][slot + 16 + 4 * g4]);
                fold_tile(
                    st, k, v, kf, vf, [&]() { load_k(t + 1); },
                    [&](float(&x)[8], uint32_t(&w)[2][8]) {
                        const uint32_t keys = (uint32_t)(seen >> slot);
                        if (keys != 0xffffffffu) hide_empty(x, w, keys >> (4 * g4));
                        const uint32_t two[4] = {r0.x, r0.y, r1.x, r1.y};
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (!(two[i >> 1] & (i & 1 ? bit << 16 : bit))) x[i] = SQ_NEG_INF;
                    });
                load_v(t + 1);
                if (even && t + 2 < tiles) list_scales(buf ^ 1);
            }
        }
        // Is a result that a row may have of another row's keys a NaN?
        bool nan = st.l != st.l;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) nan = nan || st.o[i][k] != st.o[i][k];
        hand_over(st, columns, wave, s_out, s_ml);
        const bool again = __syncthreads_or(only < 0 && nan && c16 < columns);
        const int from = only < 0 ? 0 : only * a.g, n = only < 0 ? columns : a.g;
        for (int i = threadIdx.x; i < n * D; i += 256) {
            const int column = from + (i >> 7), d = i & 127;
            store_partial(a.part + ((size_t)unit * 16 + column) * PART_STRIDE, d, join(s_out, s_ml, column, d));
        }
        __syncthreads();
        if (only < 0 && !again) break;
    }
}

void launch_decode_q8_shared(const DecodeQ8Args &a, bool wide, hipEvent_t ev0, hipEvent_t ev1, hipStream_t s)
{
    const int grid = (a.H * a.groups * a.parts + 7) / 8 * 8;
    // Where a head has one group of rows, nothing is read twice: past the caches, if the context is more than they hold (16 sequences over
    // 32 heads of 32K keys 70 -> 63 us; 40 sequences, three groups, the other way round, 40 -> 45).
    const bool once = a.groups == 1 && streams((size_t)a.H * a.L * D * 2);
    auto *kernel = wide ? (once ? decode_q8_shared_kernel<true, true> : decode_q8_shared_kernel<true, false>)
                        : (once ? decode_q8_shared_kernel<false, true> : decode_q8_shared_kernel<false, false>);
    if (ev0) hipExtLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, s, ev0, ev1, 0, a);
    else hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, s, a);
}

}  // namespace sq
