// Embedding lookup y[i] = scale w[t_i] and its gradient by token, grads[r][t] = scale * sum of the
// rows dy[i] of shard r whose token is t.
#include "device_common.h"
#include "internal.h"

#include <algorithm>

namespace mtx {

template <typename TW, typename TY>
__global__ __launch_bounds__(256) void embed_fwd_kernel(const TW* __restrict__ w, int V, int D,
                                                        const int* __restrict__ tok, long long n,
                                                        int pad, float scale, TY* __restrict__ y,
                                                        long long ldy)
{
    for (long long i = blockIdx.x; i < n; i += gridDim.x) {
        const int t = tok[i];
        const bool in = t >= 0 && t < V;
        const bool zero = pad >= 0 && t == pad;
        const TW* row = w + (long long)(in ? t : 0) * D;
        for (int d = threadIdx.x; d < D; d += 256) {
            const float v = zero ? 0.f : in ? scale * to_f32<TW>(row[d]) : __builtin_nanf("");
            y[i * ldy + d] = from_f32<TY>(v);
        }
    }
}

hipError_t embed_fwd(const void* w, Dt wt, int V, int D, const int* tok, long long n, int pad,
                     float scale, void* y, Dt yt, long long ldy, hipStream_t s)
{
    if (n == 0) return hipSuccess;
    const dim3 grid((unsigned)std::min<long long>(n, 65536));
    auto go = [&](auto tw, auto ty) {
        using TW = decltype(tw);
        using TY = decltype(ty);
        hipLaunchKernelGGL((embed_fwd_kernel<TW, TY>), grid, dim3(256), 0, s,
                           static_cast<const TW*>(w), V, D, tok, n, pad, scale,
                           static_cast<TY*>(y), ldy);
    };
    if (wt == DT_F32) yt == DT_F32 ? go(float(), float()) : go(float(), bf16_t());
    else yt == DT_F32 ? go(bf16_t(), float()) : go(bf16_t(), bf16_t());
    return hipGetLastError();
}

// One block per (row t, shard r): the shard's tokens are walked in order.
template <typename T>
__global__ __launch_bounds__(256) void embed_bwd_kernel(const int* __restrict__ tok, long long n,
                                                        const T* __restrict__ dy, long long lddy,
                                                        int D, int pad, float scale,
                                                        float* __restrict__ grads, long long ld,
                                                        bool accumulate)
{
    const int t = blockIdx.x, r = blockIdx.y;
    float* out = grads + (long long)r * ld + (long long)t * D;
    tok += r * n;
    dy += r * n * lddy;
    __shared__ int match[256];
    for (int d0 = 0; d0 < D; d0 += 256) {
        const int d = d0 + threadIdx.x;
        float acc = 0.f;
        bool any = false;
        for (long long i0 = 0; i0 < n; i0 += 256) {
            const long long i = i0 + threadIdx.x;
            const int m = i < n && tok[i] == t && t != pad;
            match[threadIdx.x] = m;
            if (__syncthreads_or(m)) {
                any = true;
                for (int j = 0; j < 256; ++j)
                    if (match[j] && d < D) acc += to_f32<T>(dy[(i0 + j) * lddy + d]);
            }
            __syncthreads();
        }
        if (d >= D) continue;
        if (!accumulate) out[d] = scale * acc;
        else if (any) out[d] += scale * acc;
    }
}

size_t embed_bwd_bytes(long long n, int R, int V, int D) { return 256; }

hipError_t embed_bwd(const int* tok, long long n, int R, const void* dy, Dt dt, long long lddy,
                     int V, int D, int pad, float scale, float* grads, long long ld,
                     bool accumulate, void* ws, hipStream_t s)
{
    const dim3 grid(V, R);
    if (dt == DT_F32)
        hipLaunchKernelGGL((embed_bwd_kernel<float>), grid, dim3(256), 0, s, tok, n,
                           static_cast<const float*>(dy), lddy, D, pad, scale, grads, ld,
                           accumulate);
    else
        hipLaunchKernelGGL((embed_bwd_kernel<bf16_t>), grid, dim3(256), 0, s, tok, n,
                           static_cast<const bf16_t*>(dy), lddy, D, pad, scale, grads, ld,
                           accumulate);
    return hipGetLastError();
}

}  // namespace mtx
