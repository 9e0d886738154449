// The end of a residual block and the norm before the next one, in one pass over the rows:
//   u = norm(x) post_w + post_b (or x);  H = h + scale gate u;  y = norm(H) pre_w + pre_b
// with RMS or layer norm over the D elements of a row, and its gradients.  With H^ = (H - mean) r,
//   dH = dh_out + r (dy pre_w - [mean(dy pre_w)] - H^ mean(dy pre_w H^))     ([]: layer norm)
//   dh = dH;  du = scale gate dH;  dx likewise through x^ = (x - mean) r
//   d_pre_w = sum dy H^, d_pre_b = sum dy, d_post_w = sum du x^, d_post_b = sum du,
//   d_gate = scale sum dH u.
// Statistics and sums are fp32; only h_out, y, dh and dx are rounded to the tensors' type.
#include "device_common.h"
#include "internal.h"

#include <algorithm>

namespace mtx {

__device__ __forceinline__ float block_sum(float v, float* red)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

// One block per row; the row of H is kept in LDS in fp32 (at most 64 KB).
template <typename T>
__global__ __launch_bounds__(256) void norm_fwd_kernel(BlockNorm b, const T* h, const T* x,
                                                       T* h_out, T* y, float* stats)
{
    extern __shared__ float row[];
    __shared__ float red[4];
    const long long i = blockIdx.x;
    const int D = b.D;
    const float inv_d = 1.0f / (float)D;
    const float* gate = b.gate ? b.gate + (b.gate_rows ? i / b.gate_rows : 0) * D : nullptr;
    float mean = 0.f, r = 1.f;
    if (x && b.post_w) {
        if (b.layer) {
            float s = 0.f;
            for (int d = threadIdx.x; d < D; d += 256) s += to_f32<T>(x[i * b.ld_x + d]);
            mean = block_sum(s, red) * inv_d;
        }
        float q = 0.f;
        for (int d = threadIdx.x; d < D; d += 256) {
            const float t = to_f32<T>(x[i * b.ld_x + d]) - mean;
            q = fmaf(t, t, q);
        }
        r = 1.0f / sqrtf(block_sum(q, red) * inv_d + b.eps);
        if (stats && threadIdx.x == 0) {
            stats[4 * i] = mean;
            stats[4 * i + 1] = r;
        }
    }
    float s = 0.f;
    for (int d = threadIdx.x; d < D; d += 256) {
        float v = to_f32<T>(h[i * b.ld_h + d]);
        if (x) {
            float u = to_f32<T>(x[i * b.ld_x + d]);
            if (b.post_w) {
                u = (u - mean) * r * b.post_w[d];
                if (b.post_b) u += b.post_b[d];
            }
            v = fmaf(b.scale * (gate ? gate[d] : 1.0f), u, v);
        }
        row[d] = v;
        s += v;
        if (h_out) h_out[i * b.ld_h + d] = from_f32<T>(v);
    }
    if (!y) return;
    mean = b.layer ? block_sum(s, red) * inv_d : 0.f;
    float q = 0.f;
    for (int d = threadIdx.x; d < D; d += 256) {
        const float t = row[d] - mean;
        q = fmaf(t, t, q);
    }
    r = 1.0f / sqrtf(block_sum(q, red) * inv_d + b.eps);
    if (stats && threadIdx.x == 0) {
        stats[4 * i + 2] = mean;
        stats[4 * i + 3] = r;
    }
    for (int d = threadIdx.x; d < D; d += 256) {
        float v = (row[d] - mean) * r * b.pre_w[d];
        if (b.pre_b) v += b.pre_b[d];
        y[i * b.ld_y + d] = from_f32<T>(v);
    }
}

hipError_t block_norm_fwd(const BlockNorm& b, const void* h, const void* x, void* h_out, void* y,
                          float* stats, hipStream_t s)
{
    if (b.rows == 0) return hipSuccess;
    auto go = [&](auto t) {
        using T = decltype(t);
        hipLaunchKernelGGL((norm_fwd_kernel<T>), dim3((unsigned)b.rows), dim3(256),
                           (size_t)b.D * 4, s, b, static_cast<const T*>(h),
                           static_cast<const T*>(x), static_cast<T*>(h_out), static_cast<T*>(y),
                           stats);
    };
    if (b.dt == DT_F32) go(float());
    else go(bf16_t());
    return hipGetLastError();
}

// dH (fp32, also kept in dH), dh and dx of one row per block.
template <typename T>
__global__ __launch_bounds__(256) void norm_bwd_kernel(BlockNorm b, BlockNormGrads g,
                                                       float* __restrict__ dH)
{
    __shared__ float red[4];
    const long long i = blockIdx.x;
    const int D = b.D;
    const float inv_d = 1.0f / (float)D;
    const T* H = static_cast<const T*>(g.h_out) + i * b.ld_h;
    const T* dy = static_cast<const T*>(g.dy) + i * b.ld_y;
    const T* dho = static_cast<const T*>(g.dh_out) + i * b.ld_h;
    const T* x = static_cast<const T*>(g.x) + i * b.ld_x;
    T* dh = static_cast<T*>(g.dh) + i * b.ld_h;
    T* dx = static_cast<T*>(g.dx) + i * b.ld_x;
    dH += i * D;
    float mean = 0.f, r = 0.f, c0 = 0.f, c1 = 0.f;
    if (g.dy) {
        mean = g.stats[4 * i + 2];
        r = g.stats[4 * i + 3];
        float s0 = 0.f, s1 = 0.f;
        for (int d = threadIdx.x; d < D; d += 256) {
            const float p = to_f32<T>(dy[d]) * b.pre_w[d];
            s0 += p;
            s1 = fmaf(p, (to_f32<T>(H[d]) - mean) * r, s1);
        }
        c1 = block_sum(s1, red) * inv_d;
        if (b.layer) c0 = block_sum(s0, red) * inv_d;
    }
    for (int d = threadIdx.x; d < D; d += 256) {
        float v = g.dh_out ? to_f32<T>(dho[d]) : 0.f;
        if (g.dy) {
            const float hat = (to_f32<T>(H[d]) - mean) * r;
            v += r * (to_f32<T>(dy[d]) * b.pre_w[d] - c0 - hat * c1);
        }
        dH[d] = v;
        if (g.dh) dh[d] = from_f32<T>(g.relu_h && !(to_f32<T>(H[d]) > 0.f) ? 0.f : v);
    }
    if (!g.dx) return;
    const float* gate = b.gate ? b.gate + (b.gate_rows ? i / b.gate_rows : 0) * D : nullptr;
    c0 = c1 = 0.f;
    if (b.post_w) {
        mean = g.stats[4 * i];
        r = g.stats[4 * i + 1];
        float s0 = 0.f, s1 = 0.f;
        for (int d = threadIdx.x; d < D; d += 256) {
            const float p = b.scale * (gate ? gate[d] : 1.f) * dH[d] * b.post_w[d];
            s0 += p;
            s1 = fmaf(p, (to_f32<T>(x[d]) - mean) * r, s1);
        }
        c1 = block_sum(s1, red) * inv_d;
        if (b.layer) c0 = block_sum(s0, red) * inv_d;
    }
    for (int d = threadIdx.x; d < D; d += 256) {
        float v = b.scale * (gate ? gate[d] : 1.f) * dH[d];
        if (b.post_w) v = r * (v * b.post_w[d] - c0 - (to_f32<T>(x[d]) - mean) * r * c1);
        dx[d] = from_f32<T>(v);
    }
}

// Parameter gradients: one block per 256 columns and row group (blockIdx.x), walking its rows.
// which: 0 the norms' weights and biases (a group = a shard), 1 the gate.
template <typename T>
__global__ __launch_bounds__(256) void norm_param_kernel(BlockNorm b, BlockNormGrads g,
                                                         const float* __restrict__ dH,
                                                         long long group, long long gate_ld,
                                                         int which)
{
    const int d = blockIdx.y * 256 + threadIdx.x, D = b.D;
    if (d >= D) return;
    const long long gr = blockIdx.x;
    float pw = 0.f, pb = 0.f, qw = 0.f, qb = 0.f, gt = 0.f;
    for (long long i = gr * group; i < (gr + 1) * group; ++i) {
        const float v = dH[i * D + d];
        float u = 0.f, xh = 0.f;
        if (g.x) {
            u = xh = to_f32<T>(static_cast<const T*>(g.x)[i * b.ld_x + d]);
            if (b.post_w) {
                xh = (xh - g.stats[4 * i]) * g.stats[4 * i + 1];
                u = xh * b.post_w[d] + (b.post_b ? b.post_b[d] : 0.f);
            }
        }
        if (which) {
            gt += b.scale * v * u;
            continue;
        }
        if (g.dy) {
            const float y = to_f32<T>(static_cast<const T*>(g.dy)[i * b.ld_y + d]);
            const float H = to_f32<T>(static_cast<const T*>(g.h_out)[i * b.ld_h + d]);
            pb += y;
            pw = fmaf(y, (H - g.stats[4 * i + 2]) * g.stats[4 * i + 3], pw);
        }
        if (g.x) {
            const float* gate = b.gate ? b.gate + (b.gate_rows ? i / b.gate_rows : 0) * D : nullptr;
            const float du = b.scale * (gate ? gate[d] : 1.f) * v;
            qb += du;
            qw = fmaf(du, xh, qw);
        }
    }
    const long long o = gr * g.ld + d;
    if (which) {
        g.gate[gr * gate_ld + d] = gt;
        return;
    }
    if (g.pre_w) g.pre_w[o] = pw;
    if (g.pre_b) g.pre_b[o] = pb;
    if (g.post_w) g.post_w[o] = qw;
    if (g.post_b) g.post_b[o] = qb;
}

size_t block_norm_bwd_bytes(const BlockNorm& b, int R) { return (size_t)b.rows * b.D * 4 + 256; }

hipError_t block_norm_bwd(const BlockNorm& b, int R, const BlockNormGrads& g, void* ws,
                          hipStream_t s)
{
    float* dH = static_cast<float*>(ws);
    auto go = [&](auto t) {
        using T = decltype(t);
        if (b.rows)
            hipLaunchKernelGGL((norm_bwd_kernel<T>), dim3((unsigned)b.rows), dim3(256), 0, s, b, g,
                               dH);
        const unsigned cols = (b.D + 255) / 256;
        if (g.pre_w || g.pre_b || g.post_w || g.post_b)
            hipLaunchKernelGGL((norm_param_kernel<T>), dim3(R, cols), dim3(256), 0, s, b, g, dH,
                               b.rows / R, 0LL, 0);
        const long long group = b.gate_rows ? b.gate_rows : b.rows / R;
        const long long ng = b.gate_rows ? b.rows / b.gate_rows : R;
        if (g.gate && ng)
            hipLaunchKernelGGL((norm_param_kernel<T>), dim3((unsigned)ng, cols), dim3(256), 0, s,
                               b, g, dH, group, b.gate_rows ? (long long)b.D : g.ld, 1);
    };
    if (b.dt == DT_F32) go(float());
    else go(bf16_t());
    return hipGetLastError();
}

}  // namespace mtx
