// sq_cache_append: new tokens' keys (normed and rotated) and values into the pages of an 8-bit cache, and the tokens' queries.
//
// A page is written by one workgroup per head and tensor, which holds the page's new rows in registers between the maximum and
// the rounding.  If the maximum asks for a larger scale than the page has, the same workgroup shifts the page's earlier codes.
//
// A key's code is decided at a border between two values that lie 1/8 apart, and with the f16 row, the f32 table and the f16 weight
// given exactly, 53 bits decide it as exact arithmetic does but once in some 10^14 values, where 24 bits would differ once in a
// million.  So the arithmetic is fp32 with a bound on its error: where the value less the bound and the value and the bound have
// the same code, that is the code; the others are taken again in double precision, the four tokens of a wave together (counted on the host
// over standard normal keys: one value in 5000 to 14000 is in doubt, four tokens in 9 to 28 have one, by the kind of rotation).
//
// 16384 tokens of 13 prompts, 32 query and 8 K/V heads (372 MB): 81 us, 4.6 TB/s.  Most of it are the queries, at the memory's rate.
// Keys and values wait for reads that follow one another (the sequence's length, the page and the position, the row of the table); rows,
// positions and weights are asked for without a branch between them (88 us with), and five waves a SIMD hide part of the rest (four: 3 us
// more; six, with registers in memory: 25 more; where rot_dim < 128 and a page may get more than 32 tokens, one or two are there at five).  In double precision throughout keys and values took 77 alone.  One token of a
// sequence: 3.7 us on the GPU, one of 64 sequences 4.8, a chain of the same reads; the call itself takes the calling thread 7.
#include "sq_head_row.hpp"
#include "sq_internal.hpp"

namespace sq {

namespace {

struct Piece {
    int b, block;              // sequence, index of its page
    int old, n;                // tokens of the page before, new ones
    int row;                   // first new token's row
};

// Tokens of sequence b: held before the call and appended by it (inside the capacity), first row.
__device__ __forceinline__ void sequence(const AppendArgs &a, int b, int &held, int &n, int &row)
{
    const int cap = a.max_pages * a.P;
    held = min(max(a.seq_len[b], 0), cap);
    if (a.cu) {
        row = min(max(a.cu[b], 0), a.n_tokens);
        n = max(min(a.cu[b + 1], a.n_tokens) - row, 0);
    } else {
        row = b * a.Lq;
        n = a.Lq;
    }
    n = min(n, cap - held);
}

__device__ __forceinline__ int pages_touched(int held, int n, int P) { return n > 0 ? (held + n - 1) / P - held / P + 1 : 0; }

// The `unit`-th page that the call appends to; false: there are not so many.  Every wave finds it for itself, 256 sequences at a time.
__device__ __forceinline__ bool find_piece(const AppendArgs &a, int unit, Piece &p)
{
    int b, j = 0, held, n, row;
    if (!a.cu) {
        b = unit / a.per_seq;
        j = unit - b * a.per_seq;
        sequence(a, b, held, n, row);
        if (j >= pages_touched(held, n, a.P)) return false;
    } else {
        const int lane = threadIdx.x & 63;
        int before = 0;
        for (int b0 = 0;; b0 += 256) {
            if (b0 >= a.B) return false;
            int t[4], sum = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int at = b0 + 4 * lane + k;
                sequence(a, min(at, a.B - 1), held, n, row);
                t[k] = at < a.B ? pages_touched(held, n, a.P) : 0;
                sum += t[k];
            }
            const int inc = wave_inclusive_scan(sum, lane);
            int ex = before + inc - sum;
            const unsigned long long here = __ballot(ex <= unit && unit < ex + sum);
            if (here != 0ull) {
                b = b0 + 4 * lane;
#pragma unroll
                for (int k = 0; k < 3; ++k)
                    if (b == b0 + 4 * lane + k && unit >= ex + t[k]) {
                        ex += t[k];
                        ++b;
                    }
                const int owner = __ffsll((long long)here) - 1;
                b = __builtin_amdgcn_readlane(b, owner);
                j = unit - __builtin_amdgcn_readlane(ex, owner);
                break;
            }
            before += __builtin_amdgcn_readlane(inc, 63);
        }
        sequence(a, b, held, n, row);
    }
    p.b = b;
    p.block = held / a.P + j;
    p.old = j == 0 ? held % a.P : 0;
    const int first = p.block * a.P + p.old;               // the page's first new slot
    p.n = min(a.P - p.old, held + n - first);
    p.row = row + first - held;
    return true;
}

// fp32 arithmetic of a key is off by at most 14 roundings of (|a| + |b|) max(|c|, |s|) of its pair (a, b), turned by (c, s) of any size: a
// sum of 128 squares (13 additions in a row, of which the root halves the error), the reciprocal root (a last place: two roundings), two
// products, and three roundings of the rotation.  (c, s) is a rotation times a length, so that is at most sqrt(2) times the length of the
// turned pair (u, v), and that at most |u| + |v|: 20 roundings of |u| + |v|, and as |u| + |v| is off as well, 24.
constexpr float KEY_ERROR = 1.5f / (1 << 20);

// A key's values in double precision, one pair after the other so that it takes few registers.
template <bool ADJACENT>
__device__ __forceinline__ void exact_key(float (&x)[8], h4 lo, h4 hi, h4 wa, h4 wb, bool norm, float eps, const float (&cs)[8], bool turns)
{
    double r = 1.0;
    if (norm) {
        double ss = 0.0;
#pragma unroll
        for (int i = 0; i < 4; ++i) ss += (double)(float)lo[i] * (double)(float)lo[i] + (double)(float)hi[i] * (double)(float)hi[i];
#pragma unroll
        for (int k = 8; k > 0; k >>= 1) ss += __shfl_xor(ss, k, 16);
        r = 1.0 / sqrt(ss / D + (double)eps);
    }
    auto value = [&](int i) {                               // dimension i of the lane's eight
        const double v = (double)(float)(i < 4 ? lo[i & 3] : hi[i & 3]);
        return norm ? v * r * (double)(float)(i < 4 ? wa[i & 3] : wb[i & 3]) : v;
    };
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int ia = ADJACENT ? 2 * i : i, ib = ADJACENT ? 2 * i + 1 : i + 4;
        const double a = value(ia), b = value(ib), c = cs[2 * i], s = cs[2 * i + 1];
        x[ia] = to_float_unbiased(turns ? a * c - b * s : a);
        x[ib] = to_float_unbiased(turns ? b * c + a * s : b);
        __builtin_amdgcn_sched_barrier(0);
    }
}

}  // namespace

// Tokens g, g + 16, .. of a page by 16 lanes each: T of them a thread.  Workgroups of the heads of one page, keys and values, follow one
// another: together they read the page's tokens of the projection row by row.
template <int T, bool ADJACENT, bool PARTIAL, bool STREAM>
__global__ __launch_bounds__(256, 5) void cache_append_kernel(AppendArgs a, RotaryArgs ra)
{
    const int tid = threadIdx.x, j = tid & 15, g = tid >> 4, wide = blockDim.x >> 4, waves = blockDim.x >> 6;
    __shared__ float s_max[4];
    if ((int)blockIdx.x >= a.kv_blocks) {                   // query rows: four heads of as many tokens as there are groups of 16 lanes
        const int at = blockIdx.x - a.kv_blocks, quads = (a.Hq + ROWS_AT_ONCE - 1) / ROWS_AT_ONCE, block = at / quads;
        const int quad = at - block * quads, token = block * wide + g;
        if (token >= a.n_tokens) return;
        if (a.cu && (token < a.cu[0] || token >= a.cu[a.B])) return;
        TurnRows rows;
        rows.n = min(ROWS_AT_ONCE, a.Hq - quad * ROWS_AT_ONCE);
#pragma unroll
        for (int i = 0; i < ROWS_AT_ONCE; ++i) {
            const int h = min(quad * ROWS_AT_ONCE + i, a.Hq - 1);
            rows.kind[i] = 0;
            rows.src[i] = a.q + (size_t)token * a.q_stride + (size_t)h * D;
            rows.dst[i] = a.q_out + ((size_t)token * a.Hq + h) * D;
        }
        turn_rows<ADJACENT, PARTIAL, STREAM>(rows, ra, a.positions[ra.rot_dim ? token : 0], j);
        return;
    }
    const int hv = blockIdx.x % (2 * a.H), unit = blockIdx.x / (2 * a.H);
    const bool value = hv >= a.H;
    const int h = value ? hv - a.H : hv;
    Piece p;
    if (!find_piece(a, unit, p)) return;
    // (the rows are read beside the page's number, not behind it; lanes behind the last token read it again, and store nothing)
    const int page = a.page_table[(size_t)p.b * a.max_pages + p.block];
    const bool norm = ra.weight[1] != nullptr, inexact = norm || ra.rot_dim > 0;
    const LanePieces lp = value ? LanePieces{8 * j, 8 * j + 4, false} : lane_pieces<ADJACENT, PARTIAL>(j, ra.rot_dim);
    auto token_of = [&](int i) { return p.row + min(i * 16 + g, p.n - 1); };
    auto row_of = [&](int token) {
        return (value ? a.v + (size_t)token * a.v_stride : a.k + (size_t)token * a.k_stride) + (size_t)h * D;
    };
    auto position_of = [&](int token) { return a.positions[ra.rot_dim ? token : 0]; };
    float x[T][8];
    h4 wa = {}, wb = {};
    {
        h4 lo[T], hi[T];
        float cs[T][8];
        int position[T];                                    // (first: the table's rows are waited for behind them)
#pragma unroll
        for (int i = 0; i < T; ++i) position[i] = position_of(token_of(i));
#pragma unroll
        for (int i = 0; i < T; ++i) {
            const _Float16 *src = row_of(token_of(i));
            lo[i] = *reinterpret_cast<const h4 *>(src + lp.a);
            hi[i] = *reinterpret_cast<const h4 *>(src + lp.b);
        }
        if (!value) {
            if (norm) {
                wa = *reinterpret_cast<const h4 *>(ra.weight[1] + lp.a);
                wb = *reinterpret_cast<const h4 *>(ra.weight[1] + lp.b);
            }
#pragma unroll
            for (int i = 0; i < T; ++i) load_turn(cs[i], ra, position[i], j, lp.turns);
        }
        if (page < 0 || page >= a.n_pages) return;
#pragma unroll
        for (int i = 0; i < T; ++i) {
            if (!value) norm_rotate<ADJACENT, PARTIAL>(x[i], lo[i], hi[i], wa, wb, norm, ra.eps, cs[i], lp.turns);
            else
#pragma unroll
                for (int c = 0; c < 8; ++c) x[i][c] = (float)(c < 4 ? lo[i][c & 3] : hi[i][c & 3]);
        }
    }
    const size_t ph = (size_t)page * a.H + h;
    uint8_t *codes = (value ? a.V8 : a.K8) + ph * a.P * D;
    float *scale = (value ? a.v_scale : a.k_scale) + ph;
    const float held = p.old > 0 ? *scale : 0.0f;           // the scale of the page's earlier tokens
    // One token's key, read and computed again in double precision.
    auto exactly = [&](float (&y)[8], int i) {
        const int token = token_of(i);
        const _Float16 *src = row_of(token);
        float cs[8];
        load_turn(cs, ra, position_of(token), j, lp.turns);
        exact_key<ADJACENT>(y, *reinterpret_cast<const h4 *>(src + lp.a), *reinterpret_cast<const h4 *>(src + lp.b), wa, wb, norm, ra.eps, cs,
                            lp.turns);
    };
    auto page_max = [&](float v) {
        v = wave_max(v);
        if ((tid & 63) == 0) s_max[tid >> 6] = v;
        __syncthreads();
        v = s_max[0];
        for (int i = 1; i < waves; ++i) v = fmaxf(v, s_max[i]);
        return v;
    };
    float most = 0.0f;                                      // (a maximum passes over NaN)
#pragma unroll
    for (int i = 0; i < T; ++i)
#pragma unroll
        for (int c = 0; c < 8; ++c) most = fmaxf(most, fabsf(x[i][c]));
    float amax = page_max(most);                            // (behind its barrier every thread has read the scale)
    uint32_t again = 0;                                     // tokens to be taken again in double precision, a bit each
    const auto exponent = [](float v) { return scale_exponent(__builtin_bit_cast(uint32_t, v)); };
    if (amax > 3.4e38f) {                                   // an infinity sets no scale
        most = 0.0f;
#pragma unroll
        for (int i = 0; i < T; ++i)
#pragma unroll
            for (int c = 0; c < 8; ++c) most = fmaxf(most, __builtin_bit_cast(float, finite_abs(x[i][c])));
        __syncthreads();                                    // (the first maxima have been read)
        amax = page_max(most);
    }
    // Where the largest finite value lies within its error of one's limit, it is taken exactly (|u| + |v| is at most twice the larger).
    if (!value && inexact && exponent(amax * (1.0f - 2 * KEY_ERROR)) != exponent(amax * (1.0f + 2 * KEY_ERROR))) {
        again = (1u << T) - 1;
        most = 0.0f;
#pragma unroll 1
        for (int i = 0; i < T; ++i) {
            float y[8];
            exactly(y, i);
#pragma unroll
            for (int c = 0; c < 8; ++c) most = fmaxf(most, __builtin_bit_cast(float, finite_abs(y[c])));
        }
        __syncthreads();                                    // (the maxima so far have been read)
        amax = page_max(most);
    }
    const int e = __builtin_amdgcn_readfirstlane(max(exponent(amax), exponent_holding(held)));
    const float inv = exp2_int(-e), f = held * inv;         // (f: 1 unless the scale rises or was no power of two)
    if (p.old > 0 && f != 1.0f) {
        for (int i = tid; i < p.old * (D / 16); i += blockDim.x) {
            u4v *c = reinterpret_cast<u4v *>(codes) + i;
            const u4v v = *c;
            *c = u4v{e4m3_rescale4(v.x, f), e4m3_rescale4(v.y, f), e4m3_rescale4(v.z, f), e4m3_rescale4(v.w, f)};
        }
    }
    auto store = [&](int i, u2v c) {
        if (i * 16 + g >= p.n) return;
        uint8_t *row = codes + (size_t)(p.old + i * 16 + g) * D;
        *reinterpret_cast<uint32_t *>(row + lp.a) = c.x;
        *reinterpret_cast<uint32_t *>(row + lp.b) = c.y;
    };
    if (!value && inexact) {
#pragma unroll
        for (int i = 0; i < T; ++i) {
            float less[8], more[8];
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                const float v = x[i][c] * inv;              // (an infinity or NaN is its pair's, if it was turned, and of no other value)
                const float d = (fabsf(x[i][c]) + fabsf(lp.turns ? x[i][ADJACENT ? c ^ 1 : c ^ 4] : x[i][c])) * (KEY_ERROR * inv);
                less[c] = v - d;
                more[c] = v + d;
            }
            const u2v down = e4m3_encode8(less), up = e4m3_encode8(more);
            if (down.x != up.x || down.y != up.y) again |= 1u << i;
            store(i, down);
        }
#pragma unroll 1
        for (int i = 0; i < T; ++i)                         // (what was stored where a code was in doubt is overwritten)
            if (__any(again >> i & 1)) {
                float y[8];
                exactly(y, i);
                store(i, e4m3_encode8(y, inv));
            }
    } else {
#pragma unroll
        for (int i = 0; i < T; ++i) store(i, e4m3_encode8(x[i], inv));
    }
    if (tid == 0) *scale = exp2_int(e);
}

hipError_t launch_cache_append(AppendArgs a, const RotaryArgs &ra, hipStream_t s)
{
    long long units;
    int most;                                               // new tokens that a page can get
    if (a.cu) {
        // n tokens touch at most n pages, and at most n / P + 2.  How they are dealt is not known here: the kernel is that of one sequence
        // with all of them, which gives a page that gets one token the lanes and reads of up to 64 (8 heads of 4 queries, pages of 64, us with
        // / without cu_tokens: a token of each of 64 sequences 12.6 / 3.9, of 1024 sequences 135 / 13).
        const long long some = a.B < a.n_tokens ? a.B : a.n_tokens;
        units = (long long)a.n_tokens / a.P + 2 * some;
        if (units > a.n_tokens) units = a.n_tokens;
        most = a.n_tokens;
    } else {
        a.per_seq = (a.Lq + a.P - 2) / a.P + 1;
        units = (long long)a.B * a.per_seq;
        most = a.Lq;
    }
    if (most > a.P) most = a.P;
    const int threads = most < 16 ? (most * 16 + 63) / 64 * 64 : 256;
    const long long kv = units * a.H * 2;
    const long long q = a.q ? ((long long)a.n_tokens * 16 + threads - 1) / threads * ((a.Hq + ROWS_AT_ONCE - 1) / ROWS_AT_ONCE) : 0;
    if (kv + q > 0x7fffffffll) return hipErrorInvalidConfiguration;
    a.kv_blocks = (int)kv;
    if (ra.rot_dim == 0) a.positions = a.seq_len;           // (read all the same, without a branch, and not used)
#define SQ_APPEND_1(A, P) cache_append_kernel<1, A, P, false>
#define SQ_APPEND_2(A, P) cache_append_kernel<2, A, P, false>
#define SQ_APPEND_4(A, P) cache_append_kernel<4, A, P, false>
#define SQ_APPEND_STREAM(A, P) cache_append_kernel<4, A, P, true>
    // (only the queries pass the caches, 6 us less for 16384 tokens of 32 + 8 heads; keys and values as well: 4 less.  Where no sequence
    // brings many tokens, the rows of a call are few)
    const bool stream = a.q && streams((size_t)a.n_tokens * ((size_t)a.Hq * 4 + (size_t)a.H * 6) * D);
    auto *kernel = most > 32 ? (stream ? SQ_FOR_ROTARY(ra, SQ_APPEND_STREAM) : SQ_FOR_ROTARY(ra, SQ_APPEND_4)) : most > 16 ? SQ_FOR_ROTARY(ra, SQ_APPEND_2) : SQ_FOR_ROTARY(ra, SQ_APPEND_1);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(kv + q)), dim3(threads), 0, s, a, ra);
    return hipGetLastError();
}

}  // namespace sq
