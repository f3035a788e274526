// sq_cache_append: new tokens' keys (normed and rotated) and values into the pages of an 8-bit cache, and the tokens' queries.
//
// A page is written by one workgroup per head and tensor, which holds the page's new rows in registers between the maximum and
// the rounding.  If the maximum asks for a larger scale than the page has, the same workgroup shifts the page's earlier codes.
//
// The key's arithmetic is double precision: a code is decided at a border between two values that lie 1/8 apart, and with the
// f16 row, the f32 table and the f16 weight given exactly, 53 bits decide it as exact arithmetic does but once in some 10^14
// values, where 24 bits would differ once in a million.
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

// The `unit`-th page that the call appends to; false: there are not so many.  Called by the whole workgroup.
__device__ __forceinline__ bool find_piece(const AppendArgs &a, int unit, Piece &p, int *s_scan /*[6]*/)
{
    int b, j = 0, held, n, row;
    if (!a.cu) {
        b = unit / a.per_seq;
        j = unit - b * a.per_seq;
        sequence(a, b, held, n, row);
        if (j >= pages_touched(held, n, a.P)) return false;
    } else {
        const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
        int before = 0;
        if (tid == 0) s_scan[4] = -1;
        for (int b0 = 0;; b0 += 256) {
            if (b0 >= a.B) return false;
            int t = 0;
            if (b0 + tid < a.B) {
                sequence(a, b0 + tid, held, n, row);
                t = pages_touched(held, n, a.P);
            }
            const int inc = wave_inclusive_scan(t, lane);
            __syncthreads();
            if (lane == 63) s_scan[wave] = inc;
            __syncthreads();
            int ex = before + inc - t;
            for (int w = 0; w < wave; ++w) ex += s_scan[w];
            if (ex <= unit && unit < ex + t) {
                s_scan[4] = b0 + tid;
                s_scan[5] = unit - ex;
            }
            __syncthreads();
            if (s_scan[4] >= 0) break;
            before += s_scan[0] + s_scan[1] + s_scan[2] + s_scan[3];
        }
        b = s_scan[4];
        j = s_scan[5];
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

}  // namespace

__global__ __launch_bounds__(256) void cache_append_kernel(AppendArgs a, RotaryArgs ra)
{
    const int tid = threadIdx.x, j = tid & 15, g = tid >> 4;
    __shared__ int s_scan[6];
    __shared__ uint32_t s_max[4];
    if ((int)blockIdx.x >= a.kv_blocks) {                   // query rows: four heads of 16 tokens
        const int at = blockIdx.x - a.kv_blocks, blocks = (a.n_tokens + 15) / 16, quad = at / blocks;
        const int token = (at - quad * blocks) * 16 + g;
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
        turn_rows(rows, ra, ra.rot_dim ? a.positions[token] : 0, j);
        return;
    }
    const int hv = blockIdx.x % (2 * a.H), unit = blockIdx.x / (2 * a.H);
    const int h = hv >> 1;
    const bool value = hv & 1;
    Piece p;
    if (!find_piece(a, unit, p, s_scan)) return;
    const int page = a.page_table[(size_t)p.b * a.max_pages + p.block];
    if (page < 0 || page >= a.n_pages) return;
    const size_t ph = (size_t)page * a.H + h;
    uint8_t *codes = (value ? a.V8 : a.K8) + ph * a.P * D;
    float *scale = (value ? a.v_scale : a.k_scale) + ph;

    const LanePieces lp = value ? LanePieces{8 * j, 8 * j + 4, false} : lane_pieces(j, ra.rot_dim, ra.adjacent != 0);
    float x[4][8];
    uint32_t amax = 0;
    double w[8] = {};
    if (!value && ra.weight[1]) load_pieces(w, ra.weight[1], lp);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = i * 16 + g;
        if (i * 16 >= p.n) break;
        const int token = p.row + min(t, p.n - 1);
        if (value) {
            load_pieces(x[i], a.v + (size_t)token * a.v_stride + (size_t)h * D, lp);
        } else {
            double e[8];
            float cs[8];
            load_turn(cs, ra, ra.rot_dim ? a.positions[token] : 0, j, lp.turns);
            load_pieces(e, a.k + (size_t)token * a.k_stride + (size_t)h * D, lp);
            norm_rotate<double>(e, w, ra.weight[1] != nullptr, (double)ra.eps, cs, lp.turns, ra.adjacent != 0);
#pragma unroll
            for (int c = 0; c < 8; ++c) x[i][c] = to_float_unbiased(e[c]);
        }
#pragma unroll
        for (int c = 0; c < 8; ++c) amax = max(amax, finite_abs(x[i][c]));
    }
#pragma unroll
    for (int k = 32; k > 0; k >>= 1) amax = max(amax, (uint32_t)__shfl_xor((int)amax, k));
    if ((tid & 63) == 0) s_max[tid >> 6] = amax;
    const int e_old = p.old > 0 ? exponent_of(*scale) : E4M3_EXP_MIN;
    __syncthreads();                                        // (every thread has read the scale)
    amax = max(max(s_max[0], s_max[1]), max(s_max[2], s_max[3]));
    const int e = max(scale_exponent(amax), e_old);
    if (p.old > 0 && e > e_old) {
        const float f = exp2_int(e_old - e < -126 ? -126 : e_old - e);
        for (int i = tid; i < p.old * (D / 8); i += 256) {
            u2v *c = reinterpret_cast<u2v *>(codes) + i;
            const u2v v = *c;
            *c = u2v{e4m3_rescale4(v.x, f), e4m3_rescale4(v.y, f)};
        }
    }
    const float inv = exp2_int(-e);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = i * 16 + g;
        if (t >= p.n) break;
        const u2v c = e4m3_encode8(x[i], inv);
        uint8_t *row = codes + (size_t)(p.old + t) * D;
        *reinterpret_cast<uint32_t *>(row + lp.a) = c.x;
        *reinterpret_cast<uint32_t *>(row + lp.b) = c.y;
    }
    if (tid == 0) *scale = exp2_int(e);
}

hipError_t launch_cache_append(AppendArgs a, const RotaryArgs &ra, hipStream_t s)
{
    long long units;
    if (a.cu) {
        // n tokens touch at most n pages, and at most n / P + 2
        const long long some = a.B < a.n_tokens ? a.B : a.n_tokens;
        units = (long long)a.n_tokens / a.P + 2 * some;
        if (units > a.n_tokens) units = a.n_tokens;
    } else {
        a.per_seq = (a.Lq + a.P - 2) / a.P + 1;
        units = (long long)a.B * a.per_seq;
    }
    const long long kv = units * a.H * 2, q = a.q ? ((long long)a.n_tokens + 15) / 16 * ((a.Hq + ROWS_AT_ONCE - 1) / ROWS_AT_ONCE) : 0;
    if (kv + q > 0x7fffffffll) return hipErrorInvalidConfiguration;
    if (kv + q == 0) return hipSuccess;
    a.kv_blocks = (int)kv;
    hipLaunchKernelGGL(cache_append_kernel, dim3((unsigned)(kv + q)), dim3(256), 0, s, a, ra);
    return hipGetLastError();
}

}  // namespace sq
