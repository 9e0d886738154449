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

// ---- gradient ----------------------------------------------------------------------------------
//
// Three launches, none of whose results depends on the order of atomics:
//   index   the tokens of a shard sorted by table row, stable (rows' terms keep their order);
//   gather  pieces of P sorted positions: a group of lanes adds the rows of dy of its piece, and
//           writes a table row whose terms all lie in the piece; the terms of a row at a piece's
//           edge become a partial sum.  Other groups write the rows without a token (dense form);
//   join    the partial sums of a row, in order.
// However the tokens are distributed, every group of the gather has the same work.

// Where the tokens of row t lie in the sorted order of their shard: entry of row t is
// [t mod NB][t / NB] (a block of the index launch writes its own entries next to each other).
struct RowSpan {
    int start, count;
};

struct EmbedIndex {
    const int* tok;
    int n, V, pad, lg, bins;   // NB = 1 << lg buckets of `bins` rows
    int *order, *row;          // [R][n] sorted: position in the shard, table row
    RowSpan* span;             // [R][NB][bins]
    int* valid;                // [R] tokens inside the table that are not padding
};

constexpr int kIndexWaves = 16;
constexpr int kIndexBins = 1024;   // rows of a bucket: 16 x 1024 counters are 64 KB of LDS

// Block (r, b) sorts the tokens t of shard r with t mod NB = b (interleaved, so that the frequent
// rows, which often lie side by side, spread over the blocks).  Every wave walks its own sixteenth of the
// tokens twice: first counting per row, then, with the counters turned into positions (ascending
// by row, then wave), writing.  The number of tokens in lower buckets, counted on the way, is
// where the block's part begins: blocks do not wait for one another.
__global__ __launch_bounds__(64 * kIndexWaves) void embed_index_kernel(EmbedIndex a)
{
    extern __shared__ int hist[];   // [kIndexWaves][bins]
    __shared__ int red[kIndexWaves], red2[kIndexWaves];
    const int NB = 1 << a.lg, b = blockIdx.x & (NB - 1), r = blockIdx.x >> a.lg;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int* tok = a.tok + (long long)r * a.n;
    for (int i = tid; i < kIndexWaves * a.bins; i += 64 * kIndexWaves) hist[i] = 0;
    __syncthreads();
    const int per = (a.n / (64 * kIndexWaves) + 1) * 64;
    const int i0 = min((long long)w * per, (long long)a.n), i1 = min((long long)i0 + per, (long long)a.n);
    int* mine = hist + w * a.bins;
    int lower = 0;
#pragma unroll 4
    for (int i = i0 + lane; i < i1; i += 64) {
        const int t = tok[i];
        const bool ok = (unsigned)t < (unsigned)a.V && t != a.pad;
        const int tb = t & (NB - 1);
        if (ok && tb < b) ++lower;
        if (ok && tb == b) atomicAdd(&mine[t >> a.lg], 1);
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) lower += __shfl_xor(lower, o);
    if (lane == 0) red[w] = lower;
    __syncthreads();
    int base = 0;
#pragma unroll
    for (int k = 0; k < kIndexWaves; ++k) base += red[k];
    // exclusive scan of the rows' totals; a thread takes one row (bins <= 1024)
    int total = 0;
    if (tid < a.bins)
#pragma unroll
        for (int k = 0; k < kIndexWaves; ++k) total += hist[k * a.bins + tid];
    int inc = total;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int v = __shfl_up(inc, o);
        if (lane >= o) inc += v;
    }
    if (lane == 63) red2[w] = inc;
    __syncthreads();
    int pos = base + inc - total, all = 0;
#pragma unroll
    for (int k = 0; k < kIndexWaves; ++k) {
        if (k < w) pos += red2[k];
        all += red2[k];
    }
    if (tid < a.bins) {
        a.span[(long long)blockIdx.x * a.bins + tid] = RowSpan{pos, total};
#pragma unroll
        for (int k = 0; k < kIndexWaves; ++k) {
            const int c = hist[k * a.bins + tid];
            hist[k * a.bins + tid] = pos;
            pos += c;
        }
    }
    if (b == NB - 1 && tid == 0) a.valid[r] = base + all;
    __syncthreads();
    if (!all) return;
    int* order = a.order + (long long)r * a.n;
    int* row = a.row + (long long)r * a.n;
    for (int i = i0; i < i1; i += 64) {
        const int t = i + lane < i1 ? tok[i + lane] : -1;
        const bool ok = (unsigned)t < (unsigned)a.V && t != a.pad && (t & (NB - 1)) == b;
        unsigned long long left = __ballot(ok);
        // the rows met among these 64 tokens, one after the other
        while (left) {
            const int t0 = __builtin_amdgcn_readlane(t, __builtin_ctzll(left));
            const unsigned long long same = __ballot(ok && t == t0);
            const int at = mine[t0 >> a.lg];
            if (ok && t == t0) {
                const int q = at + __popcll(same & ((1ull << lane) - 1));
                order[q] = i + lane;
                row[q] = t;
            }
            mine[t0 >> a.lg] = at + __popcll(same);   // every lane the same value
            left &= ~same;
        }
    }
}

struct EmbedGather {
    const int *order, *row;
    const RowSpan* span;
    const int* valid;
    const void* dy;
    long long lddy;
    int n, R, V, D, lg, bins, P, pieces, slices;
    float scale;
    float* grads;
    long long ld;
    bool accumulate;
    float* part;               // [R][pieces][2][Dp]
    int Dp;
    unsigned gather_blocks;    // the blocks after these write the rows without a token
};

// E values of a row of dy or of fp32: 16-byte vectors (VEC), else single elements 64 apart.
template <typename T, int E, bool VEC, int L>
__device__ __forceinline__ void load_row(const T* p, int c, int D, float (&v)[E])
{
    if constexpr (VEC) {
        constexpr int W = 16 / sizeof(T);
#pragma unroll
        for (int k = 0; k < E; k += W) {
            typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
            const u32x4 raw = *reinterpret_cast<const u32x4*>(p + c + k);
            const T* e = reinterpret_cast<const T*>(&raw);
#pragma unroll
            for (int j = 0; j < W; ++j) v[k + j] = to_f32<T>(e[j]);
        }
    } else {
#pragma unroll
        for (int k = 0; k < E; ++k) v[k] = c + k * L < D ? to_f32<T>(p[c + k * L]) : 0.f;
    }
}

template <int E, bool VEC, int L>
__device__ __forceinline__ void store_row(float* p, int c, int D, const float (&v)[E])
{
    if constexpr (VEC) {
        typedef float f32x4 __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int k = 0; k < E; k += 4)
            *reinterpret_cast<f32x4*>(p + c + k) = f32x4{v[k], v[k + 1], v[k + 2], v[k + 3]};
    } else {
#pragma unroll
        for (int k = 0; k < E; ++k)
            if (c + k * L < D) p[c + k * L] = v[k];
    }
}

// The final sum of a table row's columns.
template <int E, bool VEC, int L>
__device__ __forceinline__ void put_row(const EmbedGather& a, int r, int t, int c, float (&v)[E])
{
    float* out = a.grads + (long long)r * a.ld + (long long)t * a.D;
#pragma unroll
    for (int k = 0; k < E; ++k) v[k] *= a.scale;
    if (a.accumulate) {
        float was[E];
        load_row<float, E, VEC, L>(out, c, a.D, was);
#pragma unroll
        for (int k = 0; k < E; ++k) v[k] += was[k];
    }
    store_row<E, VEC, L>(out, c, a.D, v);
}

// A group of L lanes takes one piece and E L columns; U rows of dy are in flight at a time.
template <typename T, int E, bool VEC, int L>
__global__ __launch_bounds__(256) void embed_gather_kernel(EmbedGather a)
{
    constexpr int U = 8;
    if (blockIdx.x >= a.gather_blocks) {
        // rows without a token: each wave looks at 16 rows and clears the columns of those
        const int lane = threadIdx.x & 63;
        const long long w = (long long)(blockIdx.x - a.gather_blocks) * 4 + (threadIdx.x >> 6);
        const int per_shard = (a.V + 15) / 16;
        const int r = (int)(w / per_shard);
        if (r >= a.R) return;
        const int t0 = (int)(w % per_shard) * 16;
        const int t = t0 + (lane & 15);
        const int m = (1 << a.lg) - 1;
        bool none = false;
        if (lane < 16 && t < a.V)
            none = a.span[(((long long)r << a.lg) + (t & m)) * a.bins + (t >> a.lg)].count == 0;
        unsigned long long left = __ballot(none);
        while (left) {
            const int k = __builtin_ctzll(left);
            left &= left - 1;
            float* out = a.grads + (long long)r * a.ld + (long long)(t0 + k) * a.D;
            if constexpr (VEC) {
                typedef float f32x4 __attribute__((ext_vector_type(4)));
                for (int c = lane * 4; c < a.D; c += 256)
                    __builtin_nontemporal_store(f32x4{0.f, 0.f, 0.f, 0.f},
                                                reinterpret_cast<f32x4*>(out + c));
            } else {
                for (int c = lane; c < a.D; c += 64) out[c] = 0.f;
            }
        }
        return;
    }
    long long g = ((long long)blockIdx.x * 256 + threadIdx.x) / L;
    if (L == 64) g = __builtin_amdgcn_readfirstlane((int)g);
    const int l = threadIdx.x % L;
    const int slice = (int)(g % a.slices);
    const long long pc = g / a.slices;
    const int r = (int)(pc / a.pieces), p = (int)(pc % a.pieces);
    if (r >= a.R) return;
    const int nv = a.valid[r], p0 = p * a.P, p1 = min(p0 + a.P, nv);
    const int c = slice * (E * L) + (VEC ? l * E : l);
    if (p0 >= nv || c >= a.D) return;
    const int* order = a.order + (long long)r * a.n;
    const int* row = a.row + (long long)r * a.n;
    const T* dy = static_cast<const T*>(a.dy) + (long long)r * a.n * a.lddy;
    float* part = a.part + pc * 2 * a.Dp;
    int cur = row[p0];
    const bool from_before = p0 > 0 && row[p0 - 1] == cur;
    const int last = row[p1 - 1];
    const bool goes_on = p1 < nv && row[p1] == last;
    bool first = true;
    float acc[E];
#pragma unroll
    for (int k = 0; k < E; ++k) acc[k] = 0.f;
    auto flush = [&](bool out) {
        if (first && from_before) store_row<E, VEC, L>(part, c, a.D, acc);
        else if (out) store_row<E, VEC, L>(part + a.Dp, c, a.D, acc);
        else put_row<E, VEC, L>(a, r, cur, c, acc);
    };
    for (int j = p0; j < p1; j += U) {
        float v[U][E];
#pragma unroll
        for (int u = 0; u < U; ++u)
            load_row<T, E, VEC, L>(dy + (long long)order[min(j + u, p1 - 1)] * a.lddy, c, a.D, v[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (j + u >= p1) break;
            const int t = row[j + u];
            if (t != cur) {
                flush(false);
                cur = t;
                first = false;
#pragma unroll
                for (int k = 0; k < E; ++k) acc[k] = 0.f;
            }
#pragma unroll
            for (int k = 0; k < E; ++k) acc[k] += v[u][k];
        }
    }
    flush(goes_on);
}

// A row whose terms reach past the piece where they begin: one block per such piece and 256
// columns, whose four waves add a quarter of the partial sums each.
constexpr int kJoinCols = 256;
__global__ __launch_bounds__(256) void embed_join_kernel(EmbedGather a)
{
    __shared__ float sum[4][kJoinCols];
    const int js = (a.D + kJoinCols - 1) / kJoinCols;
    const long long pc = blockIdx.x / js;
    const int c0 = (int)(blockIdx.x % js) * kJoinCols;
    const int r = (int)(pc / a.pieces), p = (int)(pc % a.pieces);
    const int nv = a.valid[r], p0 = p * a.P, p1 = min(p0 + a.P, nv);
    if (p1 >= nv) return;
    const int* row = a.row + (long long)r * a.n;
    const int t = row[p1 - 1];
    if (row[p1] != t) return;
    const RowSpan sp = a.span[(((long long)r << a.lg) + (t & ((1 << a.lg) - 1))) * a.bins + (t >> a.lg)];
    if (sp.start < p0) return;   // begins in an earlier piece
    const int q1 = (sp.start + sp.count - 1) / a.P;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int m = q1 - p + 1, per = (m + 3) / 4;
    const int b0 = w * per, b1 = min(m, b0 + per);
    const float* part = a.part + pc * 2 * a.Dp;
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int k = b0; k < b1; ++k) {
        const float* q = k == 0 ? part + a.Dp : part + (long long)k * 2 * a.Dp;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int c = c0 + e * 64 + lane;
            if (c < a.D) acc[e] += q[c];
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[w][e * 64 + lane] = acc[e];
    __syncthreads();
    const int c = c0 + threadIdx.x;
    if (c >= a.D) return;
    float v[1] = {(sum[0][threadIdx.x] + sum[1][threadIdx.x]) +
                  (sum[2][threadIdx.x] + sum[3][threadIdx.x])};
    put_row<1, false, 1>(a, r, t, c, v);
}

// Buckets, pieces and the workspace's layout.
struct EmbedPlan {
    int lg, bins, P, pieces, Dp;
    size_t order, row, span, valid, part, bytes;
};

static EmbedPlan embed_plan(long long n, int R, int V, int D)
{
    EmbedPlan q{};
    // one block per bucket: enough of them to fill the GPU, each with rows that fit its counters
    while (q.lg < 24 && (1 << q.lg) < V &&
           ((long long)R << q.lg < 256 || ((V - 1) >> q.lg) + 1 > kIndexBins))
        ++q.lg;
    q.bins = ((V - 1) >> q.lg) + 1;
    const long long slices = (D + 511) / 512;
    q.P = (long long)R * n * slices >= 64 * 1024 ? 32 : 8;
    q.pieces = (int)((n + q.P - 1) / q.P);
    q.Dp = (D + 3) / 4 * 4;
    auto take = [&](size_t b) {
        const size_t o = q.bytes;
        q.bytes += (b + 255) / 256 * 256;
        return o;
    };
    const size_t N = (size_t)R * n;
    q.order = take(N * 4);
    q.row = take(N * 4);
    q.span = take(((size_t)R << q.lg) * q.bins * sizeof(RowSpan));
    q.valid = take((size_t)R * 4);
    q.part = take(q.pieces > 1 ? (size_t)R * q.pieces * 2 * q.Dp * 4 : 0);
    return q;
}

size_t embed_bwd_bytes(long long n, int R, int V, int D) { return embed_plan(n, R, V, D).bytes; }

template <typename T, int E, bool VEC, int L>
static void launch_gather(EmbedGather a, hipStream_t s)
{
    a.slices = (a.D + E * L - 1) / (E * L);
    const long long groups = (long long)a.R * a.pieces * a.slices;
    a.gather_blocks = (unsigned)((groups * L + 255) / 256);
    const long long fill = a.accumulate ? 0 : ((long long)a.R * ((a.V + 15) / 16) + 3) / 4;
    if (a.gather_blocks + fill)
        hipLaunchKernelGGL((embed_gather_kernel<T, E, VEC, L>),
                           dim3((unsigned)(a.gather_blocks + fill)), dim3(256), 0, s, a);
}

template <typename T>
static void launch_gather(const EmbedGather& a, hipStream_t s)
{
    constexpr int W = 16 / sizeof(T);
    auto al = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; };
    const bool vec = al(a.dy) && al(a.grads) && a.D % W == 0 && a.lddy % W == 0 && a.ld % 4 == 0;
    if (!vec) launch_gather<T, 4, false, 64>(a, s);
    else if (a.D <= 8 * W) launch_gather<T, W, true, 8>(a, s);
    else if (a.D <= 16 * W) launch_gather<T, W, true, 16>(a, s);
    else if (a.D <= 32 * W) launch_gather<T, W, true, 32>(a, s);
    else launch_gather<T, W, true, 64>(a, s);
}

hipError_t embed_bwd(const int* tok, long long n, int R, const void* dy, Dt dt, long long lddy,
                     int V, int D, int pad, float scale, float* grads, long long ld,
                     bool accumulate, void* ws, hipStream_t s)
{
    const EmbedPlan q = embed_plan(n, R, V, D);
    char* base = static_cast<char*>(ws);
    EmbedIndex x;
    x.tok = tok;
    x.n = (int)n; x.V = V; x.pad = pad; x.lg = q.lg; x.bins = q.bins;
    x.order = reinterpret_cast<int*>(base + q.order);
    x.row = reinterpret_cast<int*>(base + q.row);
    x.span = reinterpret_cast<RowSpan*>(base + q.span);
    x.valid = reinterpret_cast<int*>(base + q.valid);
    if (n == 0 && accumulate) return hipSuccess;
    hipLaunchKernelGGL(embed_index_kernel, dim3((unsigned)R << q.lg), dim3(64 * kIndexWaves),
                       (size_t)kIndexWaves * q.bins * 4, s, x);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    EmbedGather a{};
    a.order = x.order; a.row = x.row; a.span = x.span; a.valid = x.valid;
    a.dy = dy; a.lddy = lddy;
    a.n = (int)n; a.R = R; a.V = V; a.D = D;
    a.lg = q.lg; a.bins = q.bins; a.P = q.P; a.pieces = q.pieces;
    a.scale = scale; a.grads = grads; a.ld = ld; a.accumulate = accumulate;
    a.part = reinterpret_cast<float*>(base + q.part);
    a.Dp = q.Dp;
    if (dt == DT_F32) launch_gather<float>(a, s);
    else launch_gather<bf16_t>(a, s);
    e = hipGetLastError();
    if (e != hipSuccess || q.pieces <= 1) return e;
    const long long js = (D + kJoinCols - 1) / kJoinCols;
    hipLaunchKernelGGL(embed_join_kernel, dim3((unsigned)(R * q.pieces * js)), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace mtx
