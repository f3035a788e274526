// sq_kv_quantize: keys and values of a context to e4m3 codes with a scale per 64 rows, in the order of `perm`.
//
// 256 bytes read and 128 written per row.  A workgroup holds one block of 64 rows in registers between the maximum and the
// rounding, so the rows are read once.  What bounds it is the memory: 32 heads of 32768 keys and values through a permutation (809 MB)
// 130 us, 6.2 TB/s; 4 heads of 4096 (13 MB) 4.2.
#include "sq_e4m3.hpp"
#include "sq_internal.hpp"

namespace sq {

template <bool STREAM>
__global__ __launch_bounds__(256) void kv_quantize_kernel(QuantizeArgs a)
{
    const int tid = threadIdx.x, j = tid & 15, g = tid >> 4;
    const int blk = blockIdx.x % a.blocks, hv = blockIdx.x / a.blocks;
    const int which = hv % a.tensors;
    const size_t bh = hv / a.tensors;
    const _Float16 *X = a.X[which] + bh * a.L * D;
    uint8_t *codes = a.codes[which] + bh * a.L * D;
    const int32_t *perm = a.perm ? a.perm + bh * a.L : nullptr;
    const int first = blk * KV_BLOCK, n = min(KV_BLOCK, a.L - first);
    __shared__ uint32_t s_max[4];
    float x[4][8];
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = i * 16 + g;
        int src = first + min(r, n - 1);
        if (perm) src = min(max(perm[src], 0), a.L - 1);
        const h8 v = load_once<STREAM>(reinterpret_cast<const h8 *>(X + (size_t)src * D + 8 * j));
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[i][e] = (float)v[e];
            amax = max(amax, finite_abs(x[i][e]));
        }
    }
#pragma unroll
    for (int k = 32; k > 0; k >>= 1) amax = max(amax, (uint32_t)__shfl_xor((int)amax, k));
    if ((tid & 63) == 0) s_max[tid >> 6] = amax;
    __syncthreads();
    amax = max(max(s_max[0], s_max[1]), max(s_max[2], s_max[3]));
    const int e = scale_exponent(amax);
    const float inv = exp2_int(-e);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = i * 16 + g;
        if (r < n) store_once<STREAM>(reinterpret_cast<u2v *>(codes + (size_t)(first + r) * D + 8 * j), e4m3_encode8(x[i], inv));
    }
    if (tid == 0) a.scale[which][bh * a.blocks + blk] = exp2_int(e);
}

hipError_t launch_kv_quantize(const QuantizeArgs &a, int heads, hipStream_t s)
{
    auto *kernel = streams((size_t)a.L * heads * a.tensors * D * 3) ? kv_quantize_kernel<true> : kv_quantize_kernel<false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((size_t)a.blocks * heads * a.tensors)), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace sq
