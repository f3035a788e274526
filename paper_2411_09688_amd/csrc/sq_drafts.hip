// What stands around the attention of drafted tokens: sq_tree_prepare (masks and positions of trees), sq_tree_accept (the path that the
// model agrees with), sq_cache_commit (accepted rows into the pages of an 8-bit cache) and sq_cache_read (pages back to f16 rows).
#include "sq_e4m3.hpp"
#include "sq_internal.hpp"

namespace sq {

// A draft's ancestors have smaller numbers, so a thread that walks up from its draft meets the words of its mask from the last to the
// first, and holds one at a time.  16 drafts 1.8 us on the GPU, 64 trees of 256 (some 15 deep) 4.7: the walk, a read of LDS a step, and
// the calling thread takes 5.2.
__global__ __launch_bounds__(MAX_DRAFTS) void tree_prepare_kernel(TreeArgs a)
{
    __shared__ int s_parent[MAX_DRAFTS];
    const int b = blockIdx.x, t = threadIdx.x, W = (a.T + 31) / 32;
    const int n = a.n_drafts ? min(max(a.n_drafts[b], 0), a.T) : a.T;
    const int first = a.first ? a.first[b] : 0;
    if (t < a.T) s_parent[t] = a.parents[(size_t)b * a.T + t];
    __syncthreads();
    if (t >= a.T) return;
    const size_t row = (size_t)b * a.T + t;
    uint32_t *words = a.mask ? a.mask + row * W : nullptr;
    int depth = 0, word = W - 1;
    uint32_t bits = 0;
    auto leave = [&](int to) {                              // words [to + 1, word] are complete
        for (; word > to; --word) {
            if (words) words[word] = bits;
            bits = 0;
        }
    };
    if (t < n) {
        leave(t >> 5);
        bits = 1u << (t & 31);
        for (int at = t, p; p = s_parent[at], p >= 0 && p < at; at = p) {
            leave(p >> 5);
            bits |= 1u << (p & 31);
            ++depth;
        }
    }
    leave(-1);
    if (a.positions) a.positions[row] = first + depth;
}

hipError_t launch_tree_prepare(const TreeArgs &a, int B, hipStream_t s)
{
    hipLaunchKernelGGL(tree_prepare_kernel, dim3(B), dim3((a.T + 63) / 64 * 64), 0, s, a);
    return hipGetLastError();
}

// One wave per sequence: a lane holds every 64th draft and asks each step whether it is the next one; the lowest number wins.  16 drafts 1.6 us
// on the GPU, 256 trees of 64 3.0; the calling thread takes 6.2.
template <int N>
__global__ __launch_bounds__(64) void tree_accept_kernel(AcceptArgs a)
{
    __shared__ int s_target[64 * N];
    const int b = blockIdx.x, lane = threadIdx.x;
    const size_t row = (size_t)b * a.T;
    const int n = a.n_drafts ? min(max(a.n_drafts[b], 0), a.T) : a.T;
    int parent[N], token[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int t = 64 * k + lane;
        const bool there = t < n && t > 0;
        parent[k] = there ? a.parents[row + t] : -1;
        if (parent[k] >= t) parent[k] = -1;                 // not before it: no parent
        token[k] = there ? a.tokens[row + t] : 0;
        s_target[t] = t < n ? a.target[row + t] : -1;
    }
    wave_lds_sync();
    int count = 0, last = -1;
    for (int at = n > 0 ? 0 : -1; at >= 0;) {
        if (lane == 0) a.path[row + count] = at;
        ++count;
        last = s_target[at];
        int next = -1;
#pragma unroll
        for (int k = N - 1; k >= 0; --k) {
            const unsigned long long here = __ballot(parent[k] == at && token[k] == last);
            if (here != 0ull) next = 64 * k + __ffsll((long long)here) - 1;
        }
        at = next;
    }
    for (int i = count + lane; i < a.T; i += 64) a.path[row + i] = -1;
    if (lane == 0) {
        a.n_accepted[b] = count;
        if (a.next_token) a.next_token[b] = last;
        if (a.new_len) a.new_len[b] = a.seq_len[b] + count;
    }
}

hipError_t launch_tree_accept(const AcceptArgs &a, int B, hipStream_t s)
{
    auto *kernel = a.T <= 64 ? tree_accept_kernel<1> : a.T <= 256 ? tree_accept_kernel<4> : tree_accept_kernel<16>;
    hipLaunchKernelGGL(kernel, dim3(B), dim3(64), 0, s, a);
    return hipGetLastError();
}

// Accepted rows into their pages.  As in sq_cache_append a page is written by one workgroup per head and tensor, which holds its new
// rows in registers between the maximum and the rounding and shifts the page's earlier codes if the scale rises; here the rows
// are f16 and stand as they are, so every step is exact but the one rounding.
//
// What bounds it is the memory: four prompts of up to 8000 rows, 8 heads (160 MB) 29 us where the caches hold what the call before left, 33
// where they do not, 4.8 to 5.5 TB/s; eight of 32 heads (1.3 GB) past the caches 208 (221 with them).  Up to six rows of each of 16 sequences: 4.6 us on
// the GPU, a chain of reads (the length, the page, the rows), the call itself takes the calling thread 5.5.
// Tokens g, g + 16, .. of a page by 16 lanes each: N of them a thread.
template <int N, bool STREAM>
__global__ __launch_bounds__(256) void cache_commit_kernel(CommitArgs a)
{
    const int tid = threadIdx.x, j = tid & 15, g = tid >> 4, waves = blockDim.x >> 6;
    __shared__ uint32_t s_max[4];
    const int hv = blockIdx.x % (2 * a.H), unit = blockIdx.x / (2 * a.H), b = unit / a.per_seq, block0 = unit - b * a.per_seq;
    const bool value = hv >= a.H;
    const int h = value ? hv - a.H : hv;
    const int cap = a.max_pages * a.P, held = min(max(a.seq_len[b], 0), cap);
    const int all = min(a.n_rows ? min(max(a.n_rows[b], 0), a.T) : a.T, cap - held);
    const int block = held / a.P + block0;                  // the page, and its tokens: o old ones, n new, row0 the first of these
    const int o = block0 == 0 ? held % a.P : 0, first = block * a.P + o, n = min(a.P - o, held + all - first), row0 = first - held;
    if (n <= 0) return;
    const int page = a.page_table[(size_t)b * a.max_pages + block];
    if (page < 0 || page >= a.n_pages) return;
    const _Float16 *X = (value ? a.V : a.K) + ((size_t)b * a.H + h) * a.T * D;
    float x[N][8];
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        int row = row0 + min(i * 16 + g, n - 1);            // (lanes behind the last read it again, and store nothing)
        if (a.path) row = min(max(a.path[(size_t)b * a.T + row], 0), a.T - 1);
        const h8 v = load_once<STREAM>(reinterpret_cast<const h8 *>(X + (size_t)row * D + 8 * j));
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[i][e] = (float)v[e];
            amax = max(amax, finite_abs(x[i][e]));
        }
    }
    const size_t ph = (size_t)page * a.H + h;
    uint8_t *codes = (value ? a.V8 : a.K8) + ph * a.P * D;
    float *scale = (value ? a.v_scale : a.k_scale) + ph;
    const float was = o > 0 ? *scale : 0.0f;                // the scale of the page's earlier tokens
#pragma unroll
    for (int k = 32; k > 0; k >>= 1) amax = max(amax, (uint32_t)__shfl_xor((int)amax, k));
    if ((tid & 63) == 0) s_max[tid >> 6] = amax;
    __syncthreads();                                        // (behind it every thread has read the scale)
    amax = s_max[0];
    for (int w = 1; w < waves; ++w) amax = max(amax, s_max[w]);
    const int e = __builtin_amdgcn_readfirstlane(max(scale_exponent(amax), exponent_holding(was)));
    const float inv = exp2_int(-e), f = was * inv;          // (f: 1 unless the scale rises or was no power of two)
    if (o > 0 && f != 1.0f) {
        for (int i = tid; i < o * (D / 16); i += blockDim.x) {
            u4v *c = reinterpret_cast<u4v *>(codes) + i;
            const u4v v = *c;
            *c = u4v{e4m3_rescale4(v.x, f), e4m3_rescale4(v.y, f), e4m3_rescale4(v.z, f), e4m3_rescale4(v.w, f)};
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i * 16 + g < n) store_once<STREAM>(reinterpret_cast<u2v *>(codes + (size_t)(o + i * 16 + g) * D + 8 * j), e4m3_encode8(x[i], inv));
    if (tid == 0) *scale = exp2_int(e);
}

hipError_t launch_cache_commit(CommitArgs a, int B, hipStream_t s)
{
    a.per_seq = commit_pages(a.T, a.P);
    const long long blocks = (long long)B * a.per_seq * a.H * 2;
    if (blocks > 0x7fffffffll) return hipErrorInvalidConfiguration;
    const int most = a.T < a.P ? a.T : a.P, threads = commit_threads(a.T, a.P);
    const bool stream = streams((size_t)B * a.H * a.T * 6 * D);
    auto *kernel = most > 32 ? (stream ? cache_commit_kernel<4, true> : cache_commit_kernel<4, false>)
                   : most > 16 ? cache_commit_kernel<2, false> : cache_commit_kernel<1, false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(threads), 0, s, a);
    return hipGetLastError();
}

// Pages back to rows: READ_TOKENS tokens of a head and tensor per workgroup, 8 codes a lane, 16 lanes a token, so that a store of a wave
// fills lines.  A code times its scale is rounded to f16 once: by the conversion itself where the scale is a power of two, else as
// a product.
//
// What bounds it is the memory.  Four sequences of up to 8192 tokens, 32 heads, pages of 16 (654 MB): 82 us on the pages that the call before read,
// 98 to 100 on others, 6.6 TB/s (tokens a workgroup: 16 136, 32 98, 64 104, 128 112; 16 codes a lane, whose stores leave gaps in lines, 166; pages
// read past the caches as well as rows written so 101 for 82; products in fp32 and a conversion, with the test of the scales, 102 for 100).
// 500 tokens of 8 heads: 3.1 on the GPU, the calling thread takes 5.3.
template <bool STREAM>
__global__ __launch_bounds__(256) void cache_read_kernel(ReadArgs a)
{
    constexpr int N = READ_TOKENS / 16;
    const int tid = threadIdx.x, j = tid & 15, g = tid >> 4;
    const int chunk = blockIdx.x % a.chunks, bhv = blockIdx.x / a.chunks, hv = bhv % (2 * a.H), b = bhv / (2 * a.H);
    const bool value = hv >= a.H;
    const int h = value ? hv - a.H : hv;
    const int cap = a.max_pages << a.p_log, end = min(max(a.seq_len[b], 0), cap), first = a.first ? max(a.first[b], 0) : 0;
    const int n = min(a.U, max(end - first, 0));            // tokens of the sequence that are read
    if (chunk * READ_TOKENS >= n) return;
    const uint8_t *codes = value ? a.V8 : a.K8;
    const float *scales = value ? a.v_scale : a.k_scale;
    _Float16 *out = (value ? a.V : a.K) + ((size_t)b * a.H + h) * a.U * D;
    u2v c[N];
    float scale[N];
    int page[N];
    // (token behind the last: the last again, and nothing is stored)
    auto token = [&](int i) { return first + min(chunk * READ_TOKENS + i * 16 + g, n - 1); };
#pragma unroll
    for (int i = 0; i < N; ++i) page[i] = a.page_table[(size_t)b * a.max_pages + (token(i) >> a.p_log)];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const bool ok = page[i] >= 0 && page[i] < a.n_pages;
        const size_t ph = (size_t)(ok ? page[i] : 0) * a.H + h;
        c[i] = *reinterpret_cast<const u2v *>(codes + ((ph << a.p_log) + (token(i) & ((1 << a.p_log) - 1))) * D + 8 * j);
        scale[i] = scales[ph];
        if (!ok) {                                          // (no page: zeros)
            c[i] = u2v{0u, 0u};
            scale[i] = 0.0f;
        }
    }
    auto store = [&](int i, h8 y) {
        const int u = chunk * READ_TOKENS + i * 16 + g;
        if (u < n) store_once<STREAM>(reinterpret_cast<h8 *>(out + (size_t)u * D + 8 * j), y);
    };
    uint32_t other = 0;                                     // (not zero: a scale among them is negative, infinite or no power of two)
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t f = __builtin_bit_cast(uint32_t, scale[i]);
        other |= (f | (f + 0x800000u)) & 0x807fffffu;
    }
    if (__builtin_expect(__all(other == 0u), 1)) {
#pragma unroll
        for (int i = 0; i < N; ++i) store(i, codes_f16(c[i].x, c[i].y, scale[i]));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            h8 y;
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const f2v lo = __builtin_amdgcn_cvt_pk_f32_fp8(c[i][w], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(c[i][w], true);
                y[4 * w] = (_Float16)product_unbiased(lo.x, scale[i]);
                y[4 * w + 1] = (_Float16)product_unbiased(lo.y, scale[i]);
                y[4 * w + 2] = (_Float16)product_unbiased(hi.x, scale[i]);
                y[4 * w + 3] = (_Float16)product_unbiased(hi.y, scale[i]);
            }
            store(i, y);
        }
    }
}

hipError_t launch_cache_read(ReadArgs a, int B, hipStream_t s)
{
    a.chunks = (int)(((long long)a.U + READ_TOKENS - 1) / READ_TOKENS);
    const long long blocks = (long long)B * a.H * 2 * a.chunks;
    if (blocks > 0x7fffffffll) return hipErrorInvalidConfiguration;
    auto *kernel = streams((size_t)B * a.H * a.U * 6 * D) ? cache_read_kernel<true> : cache_read_kernel<false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace sq
