// Global gradient norm and clipping: norm = sqrt(sum g^2), then g * (max_norm / norm) where the norm
// exceeds max_norm.  Squares are added in double (an fp32 square overflows from |g| = 1.8e19 and a
// long fp32 sum loses the small tensors).  The first launch writes one partial sum per block; every
// block of the second adds all of them in the same order, so no third launch and no atomics are
// needed, and leaves at once where nothing is to be scaled or copied.
#include "device_common.h"
#include "internal.h"

#include <algorithm>
#include <type_traits>

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

// Every block: the norm from the partial sums, and the factor (a double: max_norm / norm may be below
// fp32's range where its products are not).
__device__ __forceinline__ double clip_factor(const double* part, int np, const ClipOut& o)
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
    return fin && norm > (double)o.max_norm ? (double)o.max_norm / norm : 1.0;
}

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// 16-byte vectors, two per thread and pass, 4 KB apart; the rows are read once (nontemporal).  The
// average is read again by the second launch; it is written through the caches, or past them where
// the rows' traffic would push it out (AVG_PAST).  The n % 4 elements left over: the grid's first
// thread.  AVG_UNALIGNED: rows or an average that start at any element (16 x 5M: unaligned vectors
// 72 us, single elements 99).  16 x 61M: 697 us, 5.95 TB/s.
enum Avg { AVG_CACHED, AVG_PAST, AVG_UNALIGNED };
template <int RT, bool EXACT, Avg HOW>
__global__ __launch_bounds__(256) void avg_sq_vec4(const float* __restrict__ grads, int Rrt,
                                                   long long n, long long ld,
                                                   float* __restrict__ avg,
                                                   double* __restrict__ part)
{
    typedef typename std::conditional<EXACT, double, float>::type A;
    constexpr int U = 2;
    __shared__ double red[4];
    const int R = RT > 0 ? RT : Rrt;
    typedef float uf32x4 __attribute__((ext_vector_type(4), aligned(4)));
    const long long n4 = n / 4;
    double acc = 0.0;
    for (long long base = (long long)blockIdx.x * 256 * U; base < n4;
         base += (long long)gridDim.x * 256 * U) {
        A s[U][4];
        bool ok[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            ok[u] = base + u * 256 + threadIdx.x < n4;
#pragma unroll
            for (int j = 0; j < 4; ++j) s[u][j] = A(0);
        }
        auto row = [&](int r) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (ok[u]) {
                    const float* p = grads + r * ld + 4 * (base + u * 256 + threadIdx.x);
                    const f32x4 x = HOW == AVG_UNALIGNED
                                        ? __builtin_nontemporal_load(reinterpret_cast<const uf32x4*>(p))
                                        : __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p));
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[u][j] = r == 0 ? (A)x[j] : s[u][j] + (A)x[j];
                }
        };
        if (RT > 0) {
#pragma unroll
            for (int r = 0; r < RT; ++r) row(r);
        } else {
            for (int r = 0; r < R; ++r) row(r);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!ok[u]) continue;
            f32x4 g;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                g[j] = (float)(s[u][j] / (A)R);
                acc = fma((double)g[j], (double)g[j], acc);
            }
            float* out = avg + 4 * (base + u * 256 + threadIdx.x);
            if (HOW == AVG_PAST) __builtin_nontemporal_store(g, reinterpret_cast<f32x4*>(out));
            else if (HOW == AVG_CACHED) *reinterpret_cast<f32x4*>(out) = g;
            else *reinterpret_cast<uf32x4*>(out) = g;
        }
    }
    if (blockIdx.x == 0 && threadIdx.x == 0)
        for (long long i = 4 * n4; i < n; ++i) {
            A s = (A)grads[i];
            for (int r = 1; r < R; ++r) s += (A)grads[(long long)r * ld + i];
            const float g = (float)(s / (A)R);
            avg[i] = g;
            acc = fma((double)g, (double)g, acc);
        }
    acc = block_sum(acc, red);
    if (threadIdx.x == 0) part[blockIdx.x] = acc;
}

// From the end of the vector to its start: what the first launch wrote last is still in the cache.
// `head` elements lie before the first aligned vector.
__global__ __launch_bounds__(256) void scale_kernel(float* __restrict__ g, long long n, int head,
                                                    const double* __restrict__ part, int np,
                                                    ClipOut o)
{
    const double f = clip_factor(part, np, o);
    if (f == 1.0) return;
    const long long step = (long long)gridDim.x * 256, n4 = (n - head) / 4;
    const long long t = (long long)blockIdx.x * 256 + threadIdx.x;
    f32x4* g4 = reinterpret_cast<f32x4*>(g + head);
#pragma unroll 2
    for (long long i = n4 - 1 - t; i >= 0; i -= step) {
        f32x4 v = g4[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = (float)(f * (double)v[j]);
        g4[i] = v;
    }
    if (t < head) g[t] = (float)(f * (double)g[t]);
    const long long rest = head + 4 * n4 + t;
    if (rest < n) g[rest] = (float)(f * (double)g[rest]);
}

template <bool EXACT>
static void launch_avg_sq(const float* grads, int R, long long n, long long ld, float* avg,
                          double* part, unsigned blocks, bool al, hipStream_t s)
{
    // (LDS that keeps five blocks to a compute unit, as in the averages without a norm)
    const size_t lds = 160 * 1024 / 5 - 1024;
    // Average, clip and update: 4 x 30M (600 MB) 230 us through the caches, 236 past them; 16 x 16M
    // (1.1 GB) 264 and 248.
    const Avg how = !al ? AVG_UNALIGNED : (double)n * (R + 1) * 4 > 768e6 ? AVG_PAST : AVG_CACHED;
    auto go = [&](auto rt) {
        constexpr int RT = decltype(rt)::value;
        auto kernel = how == AVG_PAST     ? avg_sq_vec4<RT, EXACT, AVG_PAST>
                      : how == AVG_CACHED ? avg_sq_vec4<RT, EXACT, AVG_CACHED>
                                          : avg_sq_vec4<RT, EXACT, AVG_UNALIGNED>;
        hipLaunchKernelGGL(kernel, dim3(blocks), dim3(256), lds, s, grads, R, n, ld, avg, part);
    };
    if (R == 1) go(std::integral_constant<int, 1>());
    else if (R == 2) go(std::integral_constant<int, 2>());
    else if (R == 4) go(std::integral_constant<int, 4>());
    else if (R == 8) go(std::integral_constant<int, 8>());
    else if (R == 16) go(std::integral_constant<int, 16>());
    else go(std::integral_constant<int, 0>());
}

hipError_t average_clip(const float* grads, int R, size_t n, size_t ld, bool exact, float max_norm,
                        float* avg, float* norm_out, int* nonfinite, double* part, hipStream_t s)
{
    const unsigned off = (unsigned)(reinterpret_cast<uintptr_t>(avg) & 15);
    const bool al = !off && (reinterpret_cast<uintptr_t>(grads) & 15) == 0 && (ld % 4 == 0 || R == 1);
    // at most five blocks to each of 256 compute units: more would run as a second, partly filled round
    const unsigned blocks = (unsigned)std::min<size_t>(1280, (n + 2047) / 2048);
    if (exact) launch_avg_sq<true>(grads, R, n, ld, avg, part, blocks, al, s);
    else launch_avg_sq<false>(grads, R, n, ld, avg, part, blocks, al, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    timing_split(s, "scale");
    const ClipOut o{max_norm, norm_out, nonfinite};
    const unsigned sblocks = (unsigned)std::min<size_t>(kClipBlocks, (n + 1023) / 1024);
    const int head = (int)std::min<size_t>(n, off ? (16 - off) / 4 : 0);
    hipLaunchKernelGGL(scale_kernel, dim3(sblocks), dim3(256), 0, s, avg, (long long)n, head, part,
                       (int)blocks, o);
    return hipGetLastError();
}

__device__ __forceinline__ float load_elem(const void* p, bool bf, unsigned i)
{
    return bf ? bf16_to_f32(static_cast<const bf16_t*>(p)[i]) : static_cast<const float*>(p)[i];
}

__device__ __forceinline__ float word_at(u32x4 v, bool bf, int k)
{
    if (!bf) return __uint_as_float(v[k]);
    return __uint_as_float(k % 2 ? v[k / 2] & 0xffff0000u : v[k / 2] << 16);
}

// 16 bytes at any element: a source need not be aligned where its destination is.
template <bool BF> struct AnyVec { typedef unsigned type __attribute__((ext_vector_type(4), aligned(4))); };
template <> struct AnyVec<true> { typedef unsigned type __attribute__((ext_vector_type(4), aligned(2))); };

// The elements of a chunk that belong to no whole vector of W: its head and its end.
template <class F> __device__ __forceinline__ void chunk_rest(const ClipChunk& k, unsigned end, F f)
{
    if (threadIdx.x < k.head) f(threadIdx.x);
    if (end + threadIdx.x < k.n) f(end + threadIdx.x);
}

template <bool BF> __device__ __forceinline__ double chunk_sq(const ClipChunk& k)
{
    constexpr int W = BF ? 8 : 4, U = 4;
    typedef typename AnyVec<BF>::type V;
    double acc = 0.0;
    auto add = [&](float x) { acc = fma((double)x, (double)x, acc); };
    const V* p = reinterpret_cast<const V*>(static_cast<const char*>(k.src) + k.head * (BF ? 2 : 4));
    const unsigned nv = (k.n - k.head) / W;
    for (unsigned i = threadIdx.x; i < nv; i += 256 * U) {
        u32x4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            v[u] = u32x4{0u, 0u, 0u, 0u};
            if (i + u * 256 < nv) v[u] = p[i + u * 256];
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < W; ++j) add(word_at(v[u], BF, j));
    }
    chunk_rest(k, k.head + nv * W, [&](unsigned i) { add(load_elem(k.src, BF, i)); });
    return acc;
}

__global__ __launch_bounds__(256) void list_sq_kernel(const ClipChunk* __restrict__ chunks,
                                                      int count, double* __restrict__ part)
{
    __shared__ double red[4];
    double acc = 0.0;
    ClipChunk next{};
    if ((int)blockIdx.x < count) next = chunks[blockIdx.x];
    for (int c = blockIdx.x; c < count; c += gridDim.x) {
        const ClipChunk k = next;
        if (c + (int)gridDim.x < count) next = chunks[c + gridDim.x];
        acc += k.src_bf16 ? chunk_sq<true>(k) : chunk_sq<false>(k);
    }
    acc = block_sum(acc, red);
    if (threadIdx.x == 0) part[blockIdx.x] = acc;
}

// 16 bytes of dst at a time: whole aligned vectors, next to each other in a wave, written past the
// caches (291 tensors bf16 -> fp32 at odd places of one vector, both launches: single elements
// through the caches 117 us; past them 120, half-line vectors 108, whole ones 88).
template <bool SB, bool DB>
__device__ __forceinline__ void chunk_scale(const ClipChunk& k, double f)
{
    constexpr int W = DB ? 8 : 4, U = 2;
    constexpr int SW = W * (SB ? 2 : 4) / 4;   // words of the source
    typedef unsigned pair_t __attribute__((ext_vector_type(2), aligned(2)));
    typedef typename AnyVec<SB>::type V;
    const char* p = static_cast<const char*>(k.src) + k.head * (SB ? 2 : 4);
    u32x4* o = reinterpret_cast<u32x4*>(static_cast<char*>(k.dst) + k.head * (DB ? 2 : 4));
    const unsigned nv = (k.n - k.head) / W;
    for (unsigned i = threadIdx.x; i < nv; i += 256 * U) {
        unsigned w[U][SW];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i + u * 256 >= nv) continue;
            const char* q = p + (size_t)(i + u * 256) * SW * 4;
            if constexpr (SW == 2) {
                const pair_t h = *reinterpret_cast<const pair_t*>(q);
                w[u][0] = h[0];
                w[u][1] = h[1];
            } else {
#pragma unroll
                for (int j = 0; j < SW; j += 4) {
                    const u32x4 h = *reinterpret_cast<const V*>(q + j * 4);
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[u][j + e] = h[e];
                }
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i + u * 256 >= nv) continue;
            float v[W];
#pragma unroll
            for (int j = 0; j < W; ++j)
                v[j] = (float)(f * (double)__uint_as_float(!SB     ? w[u][j]
                                                          : j % 2 ? w[u][j / 2] & 0xffff0000u
                                                                  : w[u][j / 2] << 16));
            u32x4 r;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                r[j] = DB ? f32_to_bf16(v[2 * j % W]) | (unsigned)f32_to_bf16(v[(2 * j + 1) % W]) << 16
                          : __float_as_uint(v[j]);
            __builtin_nontemporal_store(r, o + i + u * 256);
        }
    }
    chunk_rest(k, k.head + nv * W, [&](unsigned i) {
        const float g = (float)(f * (double)load_elem(k.src, SB, i));
        if (DB) static_cast<bf16_t*>(k.dst)[i] = f32_to_bf16(g);
        else static_cast<float*>(k.dst)[i] = g;
    });
}

// From the list's end to its start, as scale_kernel.
__global__ __launch_bounds__(256) void list_scale_kernel(const ClipChunk* __restrict__ chunks,
                                                         int count, bool all_in_place,
                                                         const double* __restrict__ part, int np,
                                                         ClipOut o)
{
    const double f = clip_factor(part, np, o);
    if (all_in_place && f == 1.0) return;
    for (int c = count - 1 - (int)blockIdx.x; c >= 0; c -= gridDim.x) {
        const ClipChunk k = chunks[c];
        if (!k.dst || (k.dst == k.src && f == 1.0)) continue;
        if (k.src_bf16) k.dst_bf16 ? chunk_scale<true, true>(k, f) : chunk_scale<true, false>(k, f);
        else k.dst_bf16 ? chunk_scale<false, true>(k, f) : chunk_scale<false, false>(k, f);
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
