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

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// 8 values as one or two 16-byte vectors.
template <typename T> __device__ __forceinline__ void load8(const T* p, float (&v)[8])
{
#pragma unroll
    for (int k = 0; k < 8; k += 16 / (int)sizeof(T)) {
        const u32x4 raw = *reinterpret_cast<const u32x4*>(p + k);
        const T* e = reinterpret_cast<const T*>(&raw);
#pragma unroll
        for (int j = 0; j < 16 / (int)sizeof(T); ++j) v[k + j] = to_f32<T>(e[j]);
    }
}

template <typename T> __device__ __forceinline__ void store8(T* p, const float (&v)[8])
{
#pragma unroll
    for (int k = 0; k < 8; k += 16 / (int)sizeof(T)) {
        u32x4 raw;
        T* e = reinterpret_cast<T*>(&raw);
#pragma unroll
        for (int j = 0; j < 16 / (int)sizeof(T); ++j) e[j] = from_f32<T>(v[k + j]);
        *reinterpret_cast<u32x4*>(p + k) = raw;
    }
}

// D a multiple of 8 and 16-byte aligned rows: a thread takes 8 values at a time, rpb rows to a block
// of 256 (one from D = 2048 on).  Bound by HBM, less what repeated tokens find in the caches:
// 32768 tokens x 4096 from fp32 rows to bf16 97 us (8.3 TB/s of rows read and written; one value per
// thread and access 199 us).
template <typename TW, typename TY>
__global__ __launch_bounds__(256) void embed_fwd_vec_kernel(const TW* __restrict__ w, int V, int D,
                                                            const int* __restrict__ tok,
                                                            long long n, int pad, float scale,
                                                            TY* __restrict__ y, long long ldy,
                                                            int rpb)
{
    const int units = D / 8, rr = threadIdx.x / units;
    const int u0 = rpb > 1 ? threadIdx.x - rr * units : threadIdx.x;
    if (rpb > 1 && rr >= rpb) return;
    for (long long i = (long long)blockIdx.x * rpb + (rpb > 1 ? rr : 0); i < n;
         i += (long long)gridDim.x * rpb) {
        const int t = tok[i];
        const bool in = (unsigned)t < (unsigned)V;
        const bool zero = pad >= 0 && t == pad;
        const TW* row = w + (long long)(in ? t : 0) * D;
        const float f = in ? scale : __builtin_nanf("");
        TY* out = y + i * ldy;
#pragma unroll 2
        for (int u = u0; u < units; u += 256) {
            float v[8];
            load8<TW>(row + 8 * u, v);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = zero ? 0.f : f * v[k];   // (the row may hold inf)
            store8<TY>(out + 8 * u, v);
        }
    }
}

hipError_t embed_fwd(const void* w, Dt wt, int V, int D, const int* tok, long long n, int pad,
                     float scale, void* y, Dt yt, long long ldy, hipStream_t s)
{
    if (n == 0) return hipSuccess;
    auto al = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; };
    const bool vec = D % 8 == 0 && ldy % 8 == 0 && al(w) && al(y);
    const int rpb = std::max(1, 256 / std::max(1, D / 8));
    auto go = [&](auto tw, auto ty) {
        using TW = decltype(tw);
        using TY = decltype(ty);
        if (vec)
            hipLaunchKernelGGL((embed_fwd_vec_kernel<TW, TY>),
                               dim3((unsigned)std::min<long long>((n + rpb - 1) / rpb, 1 << 22)),
                               dim3(256), 0, s, static_cast<const TW*>(w), V, D, tok, n, pad, scale,
                               static_cast<TY*>(y), ldy, rpb);
        else
            hipLaunchKernelGGL((embed_fwd_kernel<TW, TY>),
                               dim3((unsigned)std::min<long long>(n, 65536)), dim3(256), 0, s,
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
//   index   the tokens of a shard sorted by table row, stable (rows' terms keep their order), and
//           the rows without a token cleared (dense form);
//   gather  the rows of dy added in sorted order, blocks of equally many positions whatever the
//           tokens are; rows at the edge of a block become partial sums;
//   join    the partial sums of a row, in order.

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
    float* grads;              // rows without a token are cleared (null: left)
    long long ld;
    int D;
    bool vec;                  // grads rows take 16-byte stores
};

constexpr int kIndexWaves = 16;
constexpr int kIndexBins = 512;   // rows of a bucket: 16 x 512 counters are 32 KB of LDS

// Block (r, b) sorts the tokens t of shard r with t mod NB = b (interleaved, so that the frequent
// rows, which often lie side by side, spread over the blocks).  Every wave walks its own sixteenth of the
// tokens twice, K loads in flight (once, where that is all of them): first counting per row,
// then, with the counters turned into positions (ascending by row, then wave), placing.  The
// number of tokens in lower buckets, counted on the way, is where the block's part begins:
// blocks do not wait for one another.
struct BlockSort {
    static constexpr int K = 32;
    const int* tok;
    int* hist;             // LDS [kIndexWaves][bins] counters, then [bins] totals of the rows
    int *red, *red2;       // LDS [kIndexWaves]
    int i0, i1, base, all, NB, b, lane, w;
    int t[K];              // the wave's last (or only) loads
    unsigned hit;          // which of them hold a token of the block

    __device__ __forceinline__ bool mine(const EmbedIndex& a, int v) const
    {
        return (unsigned)v < (unsigned)a.V && v != a.pad && (v & (NB - 1)) == b;
    }
    __device__ __forceinline__ void load(int i)
    {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (i + k * 64 >= i1) break;
            t[k] = i + k * 64 + lane < i1 ? tok[i + k * 64 + lane] : -1;
        }
    }
    // Count; on return hist holds positions, and thread q < bins the first one (pos) and the
    // number (total) of its row's tokens.
    __device__ __forceinline__ void count(const EmbedIndex& a, int& pos, int& total)
    {
        const int tid = threadIdx.x;
        for (int i = tid; i < kIndexWaves * a.bins; i += 64 * kIndexWaves) hist[i] = 0;
        __syncthreads();
        const int per = (a.n + 64 * kIndexWaves - 1) / (64 * kIndexWaves) * 64;
        i0 = min((long long)w * per, (long long)a.n);
        i1 = min((long long)i0 + per, (long long)a.n);
        int lower = 0;
        hit = 0;
        for (int i = i0; i < i1; i += 64 * K) {
            load(i);
            hit = 0;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (i + k * 64 >= i1) break;
                const bool ok = (unsigned)t[k] < (unsigned)a.V && t[k] != a.pad;
                const int m = ok ? t[k] & (NB - 1) : NB;
                lower += __popcll(__ballot(m < b));
                // (most of them hold no token of the block: a branch of the whole wave)
                if (__ballot(m == b)) {
                    hit |= 1u << k;
                    if (m == b) atomicAdd(&hist[w * a.bins + (t[k] >> a.lg)], 1);
                }
            }
        }
        if (lane == 0) red[w] = lower;
        __syncthreads();
        // exclusive scan of the rows' totals; a thread takes one row (bins <= 512)
        total = 0;
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
        base = all = 0;
        pos = inc - total;
#pragma unroll
        for (int k = 0; k < kIndexWaves; ++k) {
            base += red[k];
            if (k < w) pos += red2[k];
            all += red2[k];
        }
        if (tid < a.bins) {
            hist[kIndexWaves * a.bins + tid] = total;
            int q = pos;
#pragma unroll
            for (int k = 0; k < kIndexWaves; ++k) {
                const int c = hist[k * a.bins + tid];
                hist[k * a.bins + tid] = q;
                q += c;
            }
        }
        __syncthreads();
    }
    // put(position in the block's part, position in the shard, row) for every token of the block.
    template <class Put>
    __device__ __forceinline__ void place(const EmbedIndex& a, Put put)
    {
        int* at_row = hist + w * a.bins;
        for (int i = i0; i < i1; i += 64 * K) {
            if (i1 - i0 > 64 * K) {
                load(i);
                hit = ~0u;
            }
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (i + k * 64 >= i1) break;
                if (!(hit >> k & 1)) continue;
                const bool ok = mine(a, t[k]);
                unsigned long long left = __ballot(ok);
                // the rows met among these 64 tokens, one after the other
                while (left) {
                    const int t0 = __builtin_amdgcn_readlane(t[k], __builtin_ctzll(left));
                    const unsigned long long same = __ballot(ok && t[k] == t0);
                    const int at = at_row[t0 >> a.lg];
                    if (ok && t[k] == t0)
                        put(at + __popcll(same & ((1ull << lane) - 1)), i + k * 64 + lane, t0);
                    at_row[t0 >> a.lg] = at + __popcll(same);   // every lane the same value
                    left &= ~same;
                }
            }
        }
    }
};

__device__ __forceinline__ void block_sort_init(BlockSort& k, const EmbedIndex& a, int* hist,
                                                int (&red)[2][kIndexWaves], int& r)
{
    k.NB = 1 << a.lg;
    k.b = blockIdx.x & (k.NB - 1);
    r = blockIdx.x >> a.lg;
    k.lane = threadIdx.x & 63;
    k.w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    k.tok = a.tok + (long long)r * a.n;
    k.hist = hist;
    k.red = red[0];
    k.red2 = red[1];
}

// A wave clears a row of the table's gradient.
__device__ __forceinline__ void clear_row(float* out, int D, bool vec, int lane)
{
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    if (vec)
        for (int c = lane * 4; c < D; c += 256)
            *reinterpret_cast<f32x4*>(out + c) = f32x4{0.f, 0.f, 0.f, 0.f};
    else
        for (int c = lane; c < D; c += 64) out[c] = 0.f;
}

__global__ __launch_bounds__(64 * kIndexWaves) void embed_index_kernel(EmbedIndex a)
{
    extern __shared__ int hist[];
    __shared__ int red[2][kIndexWaves];
    BlockSort k;
    int r, pos, total;
    block_sort_init(k, a, hist, red, r);
    k.count(a, pos, total);
    if ((int)threadIdx.x < a.bins)
        a.span[(long long)blockIdx.x * a.bins + threadIdx.x] = RowSpan{k.base + pos, total};
    if (k.b == k.NB - 1 && threadIdx.x == 0) a.valid[r] = k.base + k.all;
    int* order = a.order + (long long)r * a.n + k.base;
    int* row = a.row + (long long)r * a.n + k.base;
    if (k.all)
        k.place(a, [&](int q, int i, int t) {
            order[q] = i;
            row[q] = t;
        });
    if (!a.grads) return;
    // the block's rows without a token
    for (int q = k.w; q < a.bins; q += kIndexWaves) {
        const int t = (q << a.lg) + k.b;
        if (t < a.V && !hist[kIndexWaves * a.bins + q])
            clear_row(a.grads + (long long)r * a.ld + (long long)t * a.D, a.D, a.vec, k.lane);
    }
}

struct EmbedGather {
    const int *order, *row;
    const RowSpan* span;
    const int* valid;
    const void* dy;
    long long lddy;
    int n, R, V, D, lg, bins;
    int P, BP, pieces, slices; // positions of a group, of a block; blocks along a shard; along D
    long long piece0;          // the launch's first piece of all shards'
    float scale;
    float* grads;
    long long ld;
    bool accumulate;
    float* part;               // [R][pieces][2][Dp]
    int Dp;
};

// E values of a row of dy or of fp32: 16-byte vectors (VEC), else single elements L apart.
template <typename T, int E, bool VEC, int L>
__device__ __forceinline__ void load_row(const T* p, int c, int D, float (&v)[E])
{
    if constexpr (VEC) {
        constexpr int W = 16 / sizeof(T);
#pragma unroll
        for (int k = 0; k < E; k += W) {
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

// A block takes kGroups pieces of P positions in a row and E L columns, a group of L lanes one piece,
// U rows of dy in flight at a time.  A row of the table whose terms all lie in one group's
// piece is written by the group; the sums at a group's edges meet in LDS, where they are joined in
// order; what reaches over the block's edges becomes a partial sum of the block: slot 0 the
// row that began in an earlier block, slot 1 one that begins here and goes on.
constexpr int kGroups = 8;
template <typename T, int E, bool VEC, int L>
__global__ __launch_bounds__(kGroups * L) void embed_gather_kernel(EmbedGather a)
{
    constexpr int U = 8, G = kGroups, W = E * L;
    // per group: the sum of a row that began earlier (head), and of one that goes on (tail)
    __shared__ float edge[G][2][W];
    __shared__ int edge_row[G][2];   // their rows, -1: none
    __shared__ int head_ends[G];     // the head's row ends in the group
    const int slice = (int)(blockIdx.x % a.slices);
    const long long pc = a.piece0 + blockIdx.x / a.slices;
    const int r = (int)(pc / a.pieces), p = (int)(pc % a.pieces);
    const int nv = a.valid[r];
    const int b0 = p * G * a.P;
    if (b0 >= nv) return;
    int grp = threadIdx.x / L;
    if (L == 64) grp = __builtin_amdgcn_readfirstlane(grp);
    const int l = threadIdx.x % L;
    const int cl = VEC ? l * E : l;           // column in the block's slice
    const int c = slice * W + cl;
    const int* order = a.order + (long long)r * a.n;
    const int* row = a.row + (long long)r * a.n;
    const T* dy = static_cast<const T*>(a.dy) + (long long)r * a.n * a.lddy;
    const int p0 = b0 + grp * a.P, p1 = min(p0 + a.P, nv);
    if (l == 0) edge_row[grp][0] = edge_row[grp][1] = -1;
    if (p0 < nv) {
        int cur = row[p0];
        const bool from_before = p0 > 0 && row[p0 - 1] == cur;
        const bool goes_on = p1 < nv && row[p1] == row[p1 - 1];
        bool first = true;
        float acc[E];
#pragma unroll
        for (int k = 0; k < E; ++k) acc[k] = 0.f;
        auto flush = [&](bool out) {
            const bool head = first && from_before;
            if (head || out) {
                const int k = head ? 0 : 1;
                if (l == 0) {
                    edge_row[grp][k] = cur;
                    if (head) head_ends[grp] = !out;
                }
#pragma unroll
                for (int e = 0; e < E; ++e) edge[grp][k][VEC ? cl + e : cl + e * L] = acc[e];
            } else if (c < a.D) {
                put_row<E, VEC, L>(a, r, cur, c, acc);
            }
        };
        for (int j = p0; j < p1; j += U) {
            float v[U][E];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (c < a.D)
                    load_row<T, E, VEC, L>(dy + (long long)order[min(j + u, p1 - 1)] * a.lddy, c,
                                           a.D, v[u]);
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
    __syncthreads();
    for (int q = threadIdx.x; q < W; q += kGroups * L) {
        const int col = slice * W + q;
        if (col >= a.D) break;
        float* part = a.part + pc * 2 * a.Dp + col;
        float run = 0.f;
        bool here = false;   // the running row began in this block
        int open = -1;
        for (int g = 0; g < G; ++g) {
            const int t0 = edge_row[g][0], t1 = edge_row[g][1];
            if (t0 >= 0) {
                run += edge[g][0][q];
                open = t0;
                if (head_ends[g]) {
                    if (here) {
                        float v[1] = {run};
                        put_row<1, false, 1>(a, r, t0, col, v);
                    } else {
                        part[0] = run;
                    }
                    run = 0.f;
                    open = -1;
                    here = false;
                }
            }
            if (t1 >= 0) {
                run = edge[g][1][q];
                open = t1;
                here = true;
            }
        }
        if (open >= 0) part[here ? a.Dp : 0] = run;
    }
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
    const int p0 = p * a.BP, p1 = p0 + a.BP;
    if (p1 >= a.valid[r]) return;
    const int* row = a.row + (long long)r * a.n;
    const int t = row[p1 - 1];
    if (row[p1] != t) return;
    const RowSpan sp = a.span[(((long long)r << a.lg) + (t & ((1 << a.lg) - 1))) * a.bins + (t >> a.lg)];
    if (sp.start < p0) return;   // begins in an earlier piece
    const int q1 = (sp.start + sp.count - 1) / a.BP;
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

// Few tokens (n <= kSmallTokens, at most kSmallValues of dy) take one launch: a block sorts the tokens of
// its rows into LDS, and its waves add them, a row each; rows with more than 32 terms are added by
// all waves, which take equal runs of the terms.  4 x 257 tokens, 5003 rows of 300: 19.8 us in three
// launches, 11.5 in one; 256 x 1024 added to what is there 17 and 10.  Past the limits a wave's rows one
// after the other take longer than the launches: 1000 x 300 18 and 27, 256 x 4096 17 and 22.
constexpr int kSmallTokens = 512;
constexpr long long kSmallValues = 1 << 19;
template <typename T, int E, bool VEC>
__global__ __launch_bounds__(64 * kIndexWaves) void embed_small_kernel(EmbedIndex x, EmbedGather a)
{
    constexpr int U = 8, W = E * 64, kFew = 32;
    extern __shared__ int hist[];
    __shared__ int red[2][kIndexWaves], order[kSmallTokens];
    __shared__ float sum[kIndexWaves][W];
    BlockSort k;
    int r, pos, total;
    block_sort_init(k, x, hist, red, r);
    k.count(x, pos, total);
    if (k.all) k.place(x, [&](int q, int i, int) { order[q] = i; });
    __syncthreads();
    const int* totals = hist + kIndexWaves * x.bins;
    const int* ends = hist + (kIndexWaves - 1) * x.bins;   // the last wave's counters: row ends
    const T* dy = static_cast<const T*>(a.dy) + (long long)r * a.n * a.lddy;
    const int cl = VEC ? k.lane * E : k.lane;
    auto add = [&](int j0, int j1, int c, float (&acc)[E]) {
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = 0.f;
        for (int j = j0; j < j1; j += U) {
            float v[U][E];
#pragma unroll
            for (int u = 0; u < U; ++u)
                load_row<T, E, VEC, 64>(dy + (long long)order[min(j + u, j1 - 1)] * a.lddy, c, a.D,
                                        v[u]);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (j + u < j1)
#pragma unroll
                    for (int e = 0; e < E; ++e) acc[e] += v[u][e];
        }
    };
    float acc[E];
    for (int q = k.w; q < x.bins; q += kIndexWaves) {
        const int t = (q << x.lg) + k.b, m = totals[q];
        if (t >= x.V || m > kFew) continue;
        if (m == 0) {
            if (!a.accumulate)
                clear_row(a.grads + (long long)r * a.ld + (long long)t * a.D, a.D, x.vec, k.lane);
            continue;
        }
        const int end = ends[q];
        for (int c = cl; c < a.D; c += W) {
            add(end - m, end, c, acc);
            put_row<E, VEC, 64>(a, r, t, c, acc);
        }
    }
    if (k.all <= kFew) return;
    for (int q = 0; q < x.bins; ++q) {
        const int t = (q << x.lg) + k.b, m = totals[q];
        if (m <= kFew) continue;
        const int end = ends[q], per = (m + kIndexWaves - 1) / kIndexWaves;
        const int j0 = end - m + min(m, k.w * per), j1 = min(end, j0 + per);
        for (int s0 = 0; s0 < a.D; s0 += W) {
            const int c = s0 + cl;
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] = 0.f;
            if (c < a.D) add(j0, j1, c, acc);
            __syncthreads();
#pragma unroll
            for (int e = 0; e < E; ++e) sum[k.w][VEC ? cl + e : cl + e * 64] = acc[e];
            __syncthreads();
            const int col = s0 + threadIdx.x;
            if ((int)threadIdx.x < W && col < a.D) {
                float v[1] = {0.f};
#pragma unroll
                for (int g = 0; g < kIndexWaves; ++g) v[0] += sum[g][threadIdx.x];
                put_row<1, false, 1>(a, r, t, col, v);
            }
        }
    }
}

// Buckets and the workspace's layout.
struct EmbedPlan {
    int lg, bins, Dp;
    size_t order, row, span, valid, part, bytes;
};

constexpr int kMinP = 8, kMaxP = 32;

static EmbedPlan embed_plan(long long n, int R, int V, int D)
{
    EmbedPlan q{};
    // one block per bucket: enough of them to fill the GPU, each with rows that fit its counters
    while (q.lg < 28 && (1 << q.lg) < V &&
           ((long long)R << q.lg < 256 || ((V - 1) >> q.lg) + 1 > kIndexBins))
        ++q.lg;
    q.bins = ((V - 1) >> q.lg) + 1;
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
    const size_t most = (n + kGroups * kMinP - 1) / (kGroups * kMinP);
    q.part = take(most > 1 ? (size_t)R * most * 2 * q.Dp * 4 : 0);
    return q;
}

size_t embed_bwd_bytes(long long n, int R, int V, int D) { return embed_plan(n, R, V, D).bytes; }

template <typename T, int E, bool VEC, int L>
static hipError_t launch_gather(EmbedGather a, hipStream_t s)
{
    constexpr int G = kGroups;
    a.slices = (a.D + E * L - 1) / (E * L);
    // the longest piece that still gives two blocks for every compute unit
    for (a.P = kMaxP; a.P > kMinP; a.P /= 2)
        if ((long long)a.R * ((a.n + G * a.P - 1) / (G * a.P)) * a.slices >= 512) break;
    a.BP = G * a.P;
    a.pieces = (a.n + a.BP - 1) / a.BP;
    const long long pieces = (long long)a.R * a.pieces;
    // (a launch has fewer than 2^32 threads: many shards of few tokens and wide rows take several)
    const long long most = std::max(1LL, ((1LL << 32) / (kGroups * L) - 1) / a.slices);
    for (a.piece0 = 0; a.piece0 < pieces; a.piece0 += most)
        hipLaunchKernelGGL((embed_gather_kernel<T, E, VEC, L>),
                           dim3((unsigned)(std::min(most, pieces - a.piece0) * a.slices)),
                           dim3(kGroups * L), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.pieces <= 1) return e;
    timing_split(s, "join");
    const long long js = (a.D + kJoinCols - 1) / kJoinCols;
    hipLaunchKernelGGL(embed_join_kernel, dim3((unsigned)(pieces * js)), dim3(256), 0, s, a);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_gather(const EmbedGather& a, bool vec, hipStream_t s)
{
    constexpr int W = 16 / sizeof(T);
    if (!vec) return launch_gather<T, 4, false, 64>(a, s);
    if (a.D <= 8 * W) return launch_gather<T, W, true, 8>(a, s);
    if (a.D <= 16 * W) return launch_gather<T, W, true, 16>(a, s);
    if (a.D <= 32 * W) return launch_gather<T, W, true, 32>(a, s);
    return launch_gather<T, W, true, 64>(a, s);
}

hipError_t embed_bwd(const int* tok, long long n, int R, const void* dy, Dt dt, long long lddy,
                     int V, int D, int pad, float scale, float* grads, long long ld,
                     bool accumulate, void* ws, hipStream_t s)
{
    if (n == 0 && accumulate) return hipSuccess;
    const EmbedPlan q = embed_plan(n, R, V, D);
    char* base = static_cast<char*>(ws);
    auto al = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; };
    const int W = dt == DT_F32 ? 4 : 8;
    const bool vec_out = al(grads) && D % 4 == 0 && ld % 4 == 0;
    const bool vec = vec_out && al(dy) && D % W == 0 && lddy % W == 0;
    EmbedIndex x;
    x.tok = tok;
    x.n = (int)n; x.V = V; x.pad = pad; x.lg = q.lg; x.bins = q.bins;
    x.order = reinterpret_cast<int*>(base + q.order);
    x.row = reinterpret_cast<int*>(base + q.row);
    x.span = reinterpret_cast<RowSpan*>(base + q.span);
    x.valid = reinterpret_cast<int*>(base + q.valid);
    x.grads = accumulate ? nullptr : grads;
    x.ld = ld; x.D = D; x.vec = vec_out;
    const dim3 grid((unsigned)R << q.lg), block(64 * kIndexWaves);
    const size_t lds = (size_t)(kIndexWaves + 1) * q.bins * 4;
    EmbedGather a{};
    a.order = x.order; a.row = x.row; a.span = x.span; a.valid = x.valid;
    a.dy = dy; a.lddy = lddy;
    a.n = (int)n; a.R = R; a.V = V; a.D = D;
    a.lg = q.lg; a.bins = q.bins;
    a.scale = scale; a.grads = grads; a.ld = ld; a.accumulate = accumulate;
    a.part = reinterpret_cast<float*>(base + q.part);
    a.Dp = q.Dp;
    if (n <= kSmallTokens && R * n * D <= kSmallValues) {
        if (dt == DT_F32 && vec)
            hipLaunchKernelGGL((embed_small_kernel<float, 4, true>), grid, block, lds, s, x, a);
        else if (dt == DT_F32)
            hipLaunchKernelGGL((embed_small_kernel<float, 4, false>), grid, block, lds, s, x, a);
        else if (vec)
            hipLaunchKernelGGL((embed_small_kernel<bf16_t, 8, true>), grid, block, lds, s, x, a);
        else
            hipLaunchKernelGGL((embed_small_kernel<bf16_t, 4, false>), grid, block, lds, s, x, a);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(embed_index_kernel, grid, block, lds, s, x);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    timing_split(s, "gather");
    return dt == DT_F32 ? launch_gather<float>(a, vec, s) : launch_gather<bf16_t>(a, vec, s);
}

}  // namespace mtx
