// Global gradient norm and clipping: norm = sqrt(sum g^2), then g * (max_norm / norm) where the norm
// exceeds max_norm.  Squares are added in double (an fp32 square overflows from |g| = 1.8e19 and a
// long fp32 sum loses the small tensors).  The first launch writes one partial sum per block; every
// block of the second adds all of them in the same order, so no third launch and no atomics are
// needed, and leaves at once where nothing is to be scaled or copied.
#include "device_common.h"
#include "internal.h"

#include <algorithm>

namespace mtx {

// Sum over the 256 threads of a block, the same bits in every thread.
__device__ __forceinline__ double block_sum(double v, double* red)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

struct ClipOut {
    float max_norm;
    float* norm;
    int* nonfinite;
};

// Every block: the norm from the partial sums, and the factor.
__device__ __forceinline__ float clip_factor(const double* part, int np, const ClipOut& o)
{
    __shared__ double red[4];
    double v = 0.0;
    for (int i = threadIdx.x; i < np; i += 256) v += part[i];
    const double norm = sqrt(block_sum(v, red));
    const bool fin = __builtin_isfinite(norm);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        if (o.norm) *o.norm = (float)norm;
        if (o.nonfinite) *o.nonfinite = fin ? 0 : 1;
    }
    return fin && norm > (double)o.max_norm ? (float)((double)o.max_norm / norm) : 1.0f;
}

template <bool EXACT>
__global__ __launch_bounds__(256) void avg_sq_kernel(const float* __restrict__ grads, int R,
                                                     long long n, long long ld,
                                                     float* __restrict__ avg,
                                                     double* __restrict__ part)
{
    __shared__ double red[4];
    double acc = 0.0;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n;
         i += (long long)gridDim.x * 256) {
        float g;
        if (EXACT) {
            double s = (double)grads[i];
            for (int r = 1; r < R; ++r) s += (double)grads[(long long)r * ld + i];
            g = (float)(s / (double)R);
        } else {
            float s = grads[i];
            for (int r = 1; r < R; ++r) s += grads[(long long)r * ld + i];
            g = s / (float)R;
        }
        avg[i] = g;
        acc = fma((double)g, (double)g, acc);
    }
    acc = block_sum(acc, red);
    if (threadIdx.x == 0) part[blockIdx.x] = acc;
}

__global__ __launch_bounds__(256) void scale_kernel(float* __restrict__ g, long long n,
                                                    const double* __restrict__ part, int np,
                                                    ClipOut o)
{
    const float f = clip_factor(part, np, o);
    if (f == 1.0f) return;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n;
         i += (long long)gridDim.x * 256)
        g[i] *= f;
}

hipError_t average_clip(const float* grads, int R, size_t n, size_t ld, bool exact, float max_norm,
                        float* avg, float* norm_out, int* nonfinite, double* part, hipStream_t s)
{
    const unsigned blocks = (unsigned)std::min<size_t>(kClipBlocks, (n + 255) / 256);
    if (exact)
        hipLaunchKernelGGL((avg_sq_kernel<true>), dim3(blocks), dim3(256), 0, s, grads, R,
                           (long long)n, (long long)ld, avg, part);
    else
        hipLaunchKernelGGL((avg_sq_kernel<false>), dim3(blocks), dim3(256), 0, s, grads, R,
                           (long long)n, (long long)ld, avg, part);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const ClipOut o{max_norm, norm_out, nonfinite};
    hipLaunchKernelGGL(scale_kernel, dim3(blocks), dim3(256), 0, s, avg, (long long)n, part,
                       (int)blocks, o);
    return hipGetLastError();
}

__device__ __forceinline__ float load_elem(const void* p, bool bf, unsigned i)
{
    return bf ? bf16_to_f32(static_cast<const bf16_t*>(p)[i]) : static_cast<const float*>(p)[i];
}

__global__ __launch_bounds__(256) void list_sq_kernel(const ClipChunk* __restrict__ chunks,
                                                      int count, double* __restrict__ part)
{
    __shared__ double red[4];
    double acc = 0.0;
    for (int c = blockIdx.x; c < count; c += gridDim.x) {
        const ClipChunk k = chunks[c];
        for (unsigned i = threadIdx.x; i < k.n; i += 256) {
            const double g = load_elem(k.src, k.src_bf16, i);
            acc = fma(g, g, acc);
        }
    }
    acc = block_sum(acc, red);
    if (threadIdx.x == 0) part[blockIdx.x] = acc;
}

__global__ __launch_bounds__(256) void list_scale_kernel(const ClipChunk* __restrict__ chunks,
                                                         int count, bool all_in_place,
                                                         const double* __restrict__ part, int np,
                                                         ClipOut o)
{
    const float f = clip_factor(part, np, o);
    if (all_in_place && f == 1.0f) return;
    for (int c = blockIdx.x; c < count; c += gridDim.x) {
        const ClipChunk k = chunks[c];
        if (!k.dst || (k.dst == k.src && f == 1.0f)) continue;
        for (unsigned i = threadIdx.x; i < k.n; i += 256) {
            const float g = f * load_elem(k.src, k.src_bf16, i);
            if (k.dst_bf16) static_cast<bf16_t*>(k.dst)[i] = f32_to_bf16(g);
            else static_cast<float*>(k.dst)[i] = g;
        }
    }
}

hipError_t clip_list(const ClipChunk* chunks, int count, bool all_in_place, float max_norm,
                     float* norm_out, double* part, hipStream_t s)
{
    const unsigned blocks = (unsigned)std::max(1, std::min(kClipBlocks, count));
    hipLaunchKernelGGL(list_sq_kernel, dim3(blocks), dim3(256), 0, s, chunks, count, part);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const ClipOut o{max_norm, norm_out, nullptr};
    hipLaunchKernelGGL(list_scale_kernel, dim3(blocks), dim3(256), 0, s, chunks, count,
                       all_in_place, part, (int)blocks, o);
    return hipGetLastError();
}

}  // namespace mtx
