// sq_head_norm_rotate: a projection's token-major rows normed, rotated and laid out head by head.
//
// One pass over the data and nothing else: 256 bytes read and 256 written per row of a head, and the token's 8 bytes per pair
// of the table once for all of its heads.  What bounds it is the memory: 32768 tokens of 32 + 8 + 8 heads (822 MB) 141 us,
// 5.8 TB/s, 1024 tokens of 32 + 32 + 32 heads (50 MB, which the caches hold) 9.7; a single token 4 us, a chain of three reads.
#include "sq_head_row.hpp"
#include "sq_internal.hpp"

namespace sq {

// A workgroup takes 16 consecutive tokens, 16 lanes each, and four heads: a head's rows of consecutive tokens lie side by side in the
// output.
template <bool ADJACENT, bool PARTIAL, bool STREAM>
__global__ __launch_bounds__(256) void head_rows_kernel(HeadRows hr, RotaryArgs ra, int tokens)
{
    const int heads = hr.n[0] + hr.n[1] + hr.n[2], quads = (heads + ROWS_AT_ONCE - 1) / ROWS_AT_ONCE;
    const int block = blockIdx.x / quads, quad = blockIdx.x - block * quads;
    const int j = threadIdx.x & 15, token = block * 16 + (threadIdx.x >> 4);
    if (token >= tokens) return;
    const int b = token / hr.Lq, t = token - b * hr.Lq;
    TurnRows rows;
    rows.n = min(ROWS_AT_ONCE, heads - quad * ROWS_AT_ONCE);
#pragma unroll
    for (int i = 0; i < ROWS_AT_ONCE; ++i) {
        int h = min(quad * ROWS_AT_ONCE + i, heads - 1);
        const int part = h < hr.n[0] ? 0 : h < hr.n[0] + hr.n[1] ? 1 : 2;
        h -= part == 0 ? 0 : part == 1 ? hr.n[0] : hr.n[0] + hr.n[1];
        rows.kind[i] = part;
        rows.src[i] = hr.src[part] + token * hr.stride[part] + (size_t)h * D;
        rows.dst[i] = hr.dst[part] + (((size_t)b * hr.n[part] + h) * hr.Lq + t) * D;
    }
    turn_rows<ADJACENT, PARTIAL, STREAM>(rows, ra, hr.positions[ra.rot_dim ? token : 0], j);
}

hipError_t launch_head_rows(HeadRows hr, const RotaryArgs &ra, int tokens, hipStream_t s)
{
    // (read all the same, without a branch, and not used)
    if (ra.rot_dim == 0) hr.positions = reinterpret_cast<const int32_t *>(hr.src[0] ? hr.src[0] : hr.src[1] ? hr.src[1] : hr.src[2]);
    const int heads = hr.n[0] + hr.n[1] + hr.n[2];
    const dim3 grid((unsigned)((long long)((tokens + 15) / 16) * ((heads + ROWS_AT_ONCE - 1) / ROWS_AT_ONCE)));
#define SQ_HEAD_ROWS(A, P) head_rows_kernel<A, P, false>
#define SQ_HEAD_ROWS_STREAM(A, P) head_rows_kernel<A, P, true>
    auto *kernel = streams((size_t)tokens * heads * D * 4) ? SQ_FOR_ROTARY(ra, SQ_HEAD_ROWS_STREAM) : SQ_FOR_ROTARY(ra, SQ_HEAD_ROWS);
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, hr, ra, tokens);
    return hipGetLastError();
}

}  // namespace sq
