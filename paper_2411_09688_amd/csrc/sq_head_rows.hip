// sq_head_norm_rotate: a projection's token-major rows normed, rotated and laid out head by head.
//
// One pass over the data and nothing else: 256 bytes read and 256 written per row of a head, and the token's 8 bytes per pair
// of the table once for all of its heads.
#include "sq_head_row.hpp"
#include "sq_internal.hpp"

namespace sq {

__global__ __launch_bounds__(256) void head_rows_kernel(HeadRows hr, RotaryArgs ra, long long rows)
{
    const int j = threadIdx.x & 15;
    const long long r = (long long)blockIdx.x * 16 + (threadIdx.x >> 4);
    if (r >= rows) return;
    const int heads = hr.n[0] + hr.n[1] + hr.n[2];
    const long long token = r / heads;
    int h = (int)(r - token * heads);
    const int part = h < hr.n[0] ? 0 : h < hr.n[0] + hr.n[1] ? 1 : 2;
    h -= part == 0 ? 0 : part == 1 ? hr.n[0] : hr.n[0] + hr.n[1];
    const long long b = token / hr.Lq, t = token - b * hr.Lq;
    const _Float16 *src = hr.src[part] + token * hr.stride[part] + (size_t)h * D;
    _Float16 *dst = hr.dst[part] + ((b * hr.n[part] + h) * hr.Lq + t) * D;
    if (part == 2) {
        *reinterpret_cast<u4v *>(dst + 8 * j) = *reinterpret_cast<const u4v *>(src + 8 * j);
        return;
    }
    const LanePieces lp = lane_pieces(j, ra.rot_dim, ra.adjacent != 0);
    float cs[8];
    load_turn(cs, ra, ra.rot_dim ? hr.positions[token] : 0, j, lp.turns);
    store_turned_row(dst, src, ra.weight[part], ra, lp, cs);
}

hipError_t launch_head_rows(const HeadRows &hr, const RotaryArgs &ra, int tokens, hipStream_t s)
{
    const long long rows = (long long)tokens * (hr.n[0] + hr.n[1] + hr.n[2]);
    if (rows == 0) return hipSuccess;
    hipLaunchKernelGGL(head_rows_kernel, dim3((unsigned)((rows + 15) / 16)), dim3(256), 0, s, hr, ra, rows);
    return hipGetLastError();
}

}  // namespace sq
