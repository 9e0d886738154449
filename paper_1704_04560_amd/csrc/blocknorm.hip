// The end of a residual block and the norm before the next one, in one pass over the rows:
//   u = norm(x) post_w + post_b (or x);  H = h + scale gate u;  y = norm(H) pre_w + pre_b
// with RMS or layer norm over the D elements of a row, and its gradients.  With H^ = (H - mean) r,
//   dH = dh_out + r (dy pre_w - [mean(dy pre_w)] - H^ mean(dy pre_w H^))     ([]: layer norm)
//   dh = dH;  du = scale gate dH;  dx likewise through x^ = (x - mean) r
//   d_pre_w = sum dy H^, d_pre_b = sum dy, d_post_w = sum du x^, d_post_b = sum du,
//   d_gate = scale sum dH u.
// Statistics and sums are fp32; only h_out, y, dh and dx are rounded to the tensors' type.
//
// A row is held in the registers of NT threads, 8 C elements each, so that every tensor is read
// and written once: both passes are bound by HBM.  Rows of at most 512 elements take one wave and
// need no barrier.  Elements come in 16-byte vectors where D and the strides are multiples of
// 8 and the pointers aligned (VEC), else singly, NT apart.
#include "device_common.h"
#include "internal.h"

#include <algorithm>
#include <initializer_list>

namespace mtx {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// Where a thread's element k of 8 C lies in the row.
template <int NT, bool VEC> __device__ __forceinline__ int elem(int l, int k)
{
    return VEC ? ((k / 8) * NT + l) * 8 + k % 8 : k * NT + l;
}

// A thread's elements of a row as they are stored.
template <typename T, int N, bool VEC> struct Raw {
    static constexpr int kVecs = N * (int)sizeof(T) / 16;
    u32x4 v[VEC ? kVecs : 1];
    T e[VEC ? 1 : N];
};

template <typename T, int NT, int C, bool VEC>
__device__ __forceinline__ void load_raw(const T* p, int l, int D, Raw<T, 8 * C, VEC>& o)
{
    if constexpr (VEC) {
        constexpr int per = (int)sizeof(T) / 2;   // vectors to 8 elements
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int d = (c * NT + l) * 8;
#pragma unroll
            for (int q = 0; q < per; ++q)
                o.v[c * per + q] = d < D ? reinterpret_cast<const u32x4*>(p + d)[q]
                                         : u32x4{0u, 0u, 0u, 0u};
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8 * C; ++k) o.e[k] = k * NT + l < D ? p[k * NT + l] : T(0);
    }
}

template <typename T, int N, bool VEC>
__device__ __forceinline__ float raw_at(const Raw<T, N, VEC>& o, int k)
{
    if constexpr (VEC) {
        if constexpr (sizeof(T) == 4) return __uint_as_float(o.v[k / 4][k % 4]);
        const unsigned u = o.v[k / 8][(k % 8) / 2];
        return __uint_as_float(k % 2 ? u & 0xffff0000u : u << 16);
    } else {
        return to_f32<T>(o.e[k]);
    }
}

template <typename T, int NT, int C, bool VEC>
__device__ __forceinline__ void store_row(T* p, int l, int D, const float (&v)[8 * C])
{
    if constexpr (VEC) {
        constexpr int W = 16 / (int)sizeof(T);
#pragma unroll
        for (int k = 0; k < 8 * C; k += W) {
            const int d = elem<NT, true>(l, k);
            if (d >= D) continue;
            u32x4 raw;
            T* e = reinterpret_cast<T*>(&raw);
#pragma unroll
            for (int j = 0; j < W; ++j) e[j] = from_f32<T>(v[k + j]);
            *reinterpret_cast<u32x4*>(p + d) = raw;
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8 * C; ++k)
            if (k * NT + l < D) p[k * NT + l] = from_f32<T>(v[k]);
    }
}

// Sums over the NT threads of a row, the same bits in each.  `slot` alternates between calls: a
// wave writes the slot of two calls ago only after a barrier that follows all its reads.
template <int NT, int M>
__device__ __forceinline__ void row_sum(float (&v)[M], float (&red)[2][M > 1 ? 2 : 1][16], int& slot)
{
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int o = 32; o; o >>= 1) v[m] += __shfl_xor(v[m], o);
    if constexpr (NT > 64) {
        const int wave = threadIdx.x >> 6, first = threadIdx.x / NT * (NT / 64);
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int m = 0; m < M; ++m) red[slot][m][wave] = v[m];
        __syncthreads();
#pragma unroll
        for (int m = 0; m < M; ++m) {
            v[m] = red[slot][m][first];
#pragma unroll
            for (int k = 1; k < NT / 64; ++k) v[m] += red[slot][m][first + k];
        }
        slot ^= 1;
    }
}

constexpr int block_of(int NT) { return NT < 256 ? 256 : NT; }

template <typename T, int NT, int C, bool VEC, bool LAYER>
__global__ __launch_bounds__(block_of(NT)) void norm_fwd_kernel(BlockNorm b, const T* h, const T* x,
                                                                T* h_out, T* y, float* stats)
{
    constexpr int N = 8 * C, RPB = block_of(NT) / NT;
    __shared__ float red[2][1][16];
    int slot = 0;
    const int l = threadIdx.x % NT, D = b.D;
    const float inv_d = 1.0f / (float)D;
    // (a block's rows run together: those past the end repeat the last one, storing nothing)
    const long long want = (long long)blockIdx.x * RPB + threadIdx.x / NT;
    const bool live = want < b.rows;
    const long long i = live ? want : b.rows - 1;
    Raw<T, N, VEC> rh, rx;
    load_raw<T, NT, C, VEC>(h + i * b.ld_h, l, D, rh);
    if (x) load_raw<T, NT, C, VEC>(x + i * b.ld_x, l, D, rx);
    auto norm = [&](float (&v)[N], const float* w, const float* bias, int stat) {
        float s[1], mean = 0.f;
        if constexpr (LAYER) {
            s[0] = 0.f;
#pragma unroll
            for (int k = 0; k < N; ++k) s[0] += v[k];   // (elements past D are 0)
            row_sum<NT, 1>(s, red, slot);
            mean = s[0] * inv_d;
        }
        s[0] = 0.f;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float t = LAYER && elem<NT, VEC>(l, k) >= D ? 0.f : v[k] - mean;
            s[0] = fmaf(t, t, s[0]);
        }
        row_sum<NT, 1>(s, red, slot);
        const float r = 1.0f / sqrtf(s[0] * inv_d + b.eps);
        if (stats && live && l == 0)
            *reinterpret_cast<float2*>(stats + 4 * i + stat) = make_float2(mean, r);
        Raw<float, N, VEC> rw, rb;
        load_raw<float, NT, C, VEC>(w, l, D, rw);
        if (LAYER && bias) load_raw<float, NT, C, VEC>(bias, l, D, rb);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            v[k] = (v[k] - mean) * r * raw_at(rw, k);
            if (LAYER && bias) v[k] += raw_at(rb, k);
        }
    };
    float H[N];
#pragma unroll
    for (int k = 0; k < N; ++k) H[k] = raw_at(rh, k);
    if (x) {
        float u[N];
#pragma unroll
        for (int k = 0; k < N; ++k) u[k] = raw_at(rx, k);
        if (b.post_w) norm(u, b.post_w, b.post_b, 0);
        if (b.gate) {
            Raw<float, N, VEC> rg;
            load_raw<float, NT, C, VEC>(b.gate + (b.gate_rows ? i / b.gate_rows : 0) * D, l, D, rg);
#pragma unroll
            for (int k = 0; k < N; ++k) H[k] = fmaf(b.scale * raw_at(rg, k), u[k], H[k]);
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) H[k] = fmaf(b.scale, u[k], H[k]);
        }
        if (h_out && live) store_row<T, NT, C, VEC>(h_out + i * b.ld_h, l, D, H);
    }
    if (!y) return;
    norm(H, b.pre_w, b.pre_b, 2);
    if (live) store_row<T, NT, C, VEC>(y + i * b.ld_y, l, D, H);
}

static bool al16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

static bool norm_vec(const BlockNorm& b, std::initializer_list<const void*> ptrs)
{
    bool ok = b.D % 8 == 0 && b.ld_h % 8 == 0 && b.ld_x % 8 == 0 && b.ld_y % 8 == 0 &&
              al16(b.post_w) && al16(b.post_b) && al16(b.gate) && al16(b.pre_w) && al16(b.pre_b);
    for (const void* p : ptrs) ok = ok && al16(p);
    return ok;
}

template <typename T, int NT, int C>
static void launch_fwd(const BlockNorm& b, bool vec, const void* h, const void* x, void* h_out,
                       void* y, float* stats, hipStream_t s)
{
    constexpr int RPB = block_of(NT) / NT;
    const dim3 grid((unsigned)((b.rows + RPB - 1) / RPB)), block(block_of(NT));
    const T *hh = static_cast<const T*>(h), *xx = static_cast<const T*>(x);
    T *ho = static_cast<T*>(h_out), *yy = static_cast<T*>(y);
    if (vec && b.layer)
        hipLaunchKernelGGL((norm_fwd_kernel<T, NT, C, true, true>), grid, block, 0, s, b, hh, xx, ho, yy, stats);
    else if (vec)
        hipLaunchKernelGGL((norm_fwd_kernel<T, NT, C, true, false>), grid, block, 0, s, b, hh, xx, ho, yy, stats);
    else if (b.layer)
        hipLaunchKernelGGL((norm_fwd_kernel<T, NT, C, false, true>), grid, block, 0, s, b, hh, xx, ho, yy, stats);
    else
        hipLaunchKernelGGL((norm_fwd_kernel<T, NT, C, false, false>), grid, block, 0, s, b, hh, xx, ho, yy, stats);
}

hipError_t block_norm_fwd(const BlockNorm& b, const void* h, const void* x, void* h_out, void* y,
                          float* stats, hipStream_t s)
{
    if (b.rows == 0) return hipSuccess;
    const bool vec = norm_vec(b, {h, x, h_out, y});
    auto go = [&](auto t) {
        using T = decltype(t);
        if (b.D <= 512) launch_fwd<T, 64, 1>(b, vec, h, x, h_out, y, stats, s);
        else if (b.D <= 1024) launch_fwd<T, 128, 1>(b, vec, h, x, h_out, y, stats, s);
        else if (b.D <= 2048) launch_fwd<T, 256, 1>(b, vec, h, x, h_out, y, stats, s);
        else if (b.D <= 4096) launch_fwd<T, 512, 1>(b, vec, h, x, h_out, y, stats, s);
        else if (b.D <= 8192) launch_fwd<T, 1024, 1>(b, vec, h, x, h_out, y, stats, s);
        else launch_fwd<T, 1024, 2>(b, vec, h, x, h_out, y, stats, s);
    };
    if (b.dt == DT_F32) go(float());
    else go(bf16_t());
    return hipGetLastError();
}

// ---- backward ----------------------------------------------------------------------------------
//
// A block takes rows of one shard (of one gate group, where a group is longer than that), holds
// the parameters' sums over its rows in registers, and writes them as partial sums; a second
// launch adds the blocks' partial sums of a shard (of a group) in order.

// How the rows are dealt to blocks.  Groups (a gate vector's rows, or a shard) of `group` rows are cut
// into `pieces` pieces of `chunk` rows, or `gpb` whole groups make a block.
struct NormDeal {
    long long group, groups_shard;   // rows of a group, groups of a shard
    int pieces, chunk, gpb;
    long long blocks_shard, blocks;
};

static NormDeal norm_deal(const BlockNorm& b, int R)
{
    NormDeal q{};
    const long long nb = b.rows / R;
    q.group = b.gate_rows ? b.gate_rows : nb;
    q.groups_shard = q.group ? nb / q.group : 0;
    const long long target = std::max<long long>(1, 512 / R);   // blocks of a shard
    const long long rows = std::max<long long>(1, (nb + target - 1) / target);
    q.gpb = 1;
    q.pieces = 1;
    if (q.group > rows) {
        q.pieces = (int)((q.group + rows - 1) / rows);
        q.chunk = (int)((q.group + q.pieces - 1) / q.pieces);
    } else {
        q.gpb = (int)(q.group ? std::max<long long>(1, rows / q.group) : 1);
        q.chunk = (int)q.group;
    }
    q.blocks_shard = q.pieces > 1 ? q.groups_shard * q.pieces : (q.groups_shard + q.gpb - 1) / q.gpb;
    q.blocks = q.blocks_shard * R;
    return q;
}

// planes of a block's partial sums
enum { PL_PRE_W, PL_POST_W, PL_GATE, PL_PRE_B, PL_POST_B, kPlanes };

template <typename T, int NT, int C, bool VEC, bool LAYER>
__global__ __launch_bounds__(block_of(NT)) void norm_bwd_kernel(BlockNorm b, BlockNormGrads g,
                                                                NormDeal q, float* __restrict__ part)
{
    constexpr int N = 8 * C, RPB = block_of(NT) / NT;
    __shared__ float red[2][2][16];
    __shared__ float comb[RPB > 1 ? RPB - 1 : 1][RPB > 1 ? N * NT : 1];
    int slot = 0;
    const int l = threadIdx.x % NT, rs = threadIdx.x / NT, D = b.D;
    const float inv_d = 1.0f / (float)D;
    const long long shard = blockIdx.x / q.blocks_shard, bs = blockIdx.x % q.blocks_shard;
    const long long nb = q.group * q.groups_shard;
    long long g0, g1;   // the block's groups, within the shard
    int first = 0;      // its first row within the group
    if (q.pieces > 1) {
        g0 = bs / q.pieces;
        g1 = g0 + 1;
        first = (int)(bs % q.pieces) * q.chunk;
    } else {
        g0 = bs * q.gpb;
        g1 = min(g0 + q.gpb, q.groups_shard);
    }
    const int rows = (int)max(0LL, min((long long)q.chunk, q.group - first));   // of each group
    const bool has_x = g.x != nullptr, has_y = g.dy != nullptr;
    const bool post = b.post_w != nullptr;
    float pw[N], qw[N], gt[N], pb[LAYER ? N : 1], qb[LAYER ? N : 1];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        pw[k] = qw[k] = gt[k] = 0.f;
        if (LAYER) pb[k] = qb[k] = 0.f;
    }
    // add the row slots' sums in order, into the first one's
    auto combine = [&](float (&v)[N]) {
        if constexpr (RPB > 1) {
            __syncthreads();
            if (rs)
#pragma unroll
                for (int k = 0; k < N; ++k) comb[rs - 1][k * NT + l] = v[k];
            __syncthreads();
            if (rs == 0)
#pragma unroll
                for (int o = 0; o < RPB - 1; ++o)
#pragma unroll
                    for (int k = 0; k < N; ++k) v[k] += comb[o][k * NT + l];
        }
    };
    for (long long gi = g0; gi < g1; ++gi) {
        const long long base = shard * nb + gi * q.group + first;
        const float* gate = b.gate ? b.gate + (b.gate_rows ? base / b.gate_rows : 0) * D : nullptr;
        for (int j0 = 0; j0 < rows; j0 += RPB) {
            const bool live = j0 + rs < rows;
            const long long i = base + (live ? j0 + rs : 0);
            Raw<T, N, VEC> rH, ry, ro, rx;
            Raw<float, N, VEC> rw;
            float4 st = make_float4(0.f, 0.f, 0.f, 0.f);
            if (g.stats) st = *reinterpret_cast<const float4*>(g.stats + 4 * i);
            float dH[N];
            if (has_y) {
                load_raw<T, NT, C, VEC>(static_cast<const T*>(g.h_out) + i * b.ld_h, l, D, rH);
                load_raw<T, NT, C, VEC>(static_cast<const T*>(g.dy) + i * b.ld_y, l, D, ry);
            }
            if (g.dh_out)
                load_raw<T, NT, C, VEC>(static_cast<const T*>(g.dh_out) + i * b.ld_h, l, D, ro);
            if (has_x) load_raw<T, NT, C, VEC>(static_cast<const T*>(g.x) + i * b.ld_x, l, D, rx);
#pragma unroll
            for (int k = 0; k < N; ++k) dH[k] = g.dh_out ? raw_at(ro, k) : 0.f;
            if (has_y) {
                load_raw<float, NT, C, VEC>(b.pre_w, l, D, rw);
                float s[2] = {0.f, 0.f};
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    const float p = raw_at(ry, k) * raw_at(rw, k);
                    s[0] = fmaf(p, (raw_at(rH, k) - st.z) * st.w, s[0]);
                    if (LAYER) s[1] += p;
                }
                row_sum<NT, 2>(s, red, slot);
                const float c1 = s[0] * inv_d, c0 = LAYER ? s[1] * inv_d : 0.f;
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    const float dy = raw_at(ry, k), hat = (raw_at(rH, k) - st.z) * st.w;
                    dH[k] += st.w * (dy * raw_at(rw, k) - c0 - hat * c1);
                    if (live) {
                        pw[k] = fmaf(dy, hat, pw[k]);
                        if (LAYER) pb[k] += dy;
                    }
                }
            }
            if (g.dh && live) {
                if (g.relu_h) {
                    float v[N];
#pragma unroll
                    for (int k = 0; k < N; ++k) v[k] = raw_at(rH, k) > 0.f ? dH[k] : 0.f;
                    store_row<T, NT, C, VEC>(static_cast<T*>(g.dh) + i * b.ld_h, l, D, v);
                } else {
                    store_row<T, NT, C, VEC>(static_cast<T*>(g.dh) + i * b.ld_h, l, D, dH);
                }
            }
            if (!has_x) continue;
            // du = scale gate dH; the gate's gradient is scale sum dH u
            float du[N];
            if (gate) {
                Raw<float, N, VEC> rg;
                load_raw<float, NT, C, VEC>(gate, l, D, rg);
#pragma unroll
                for (int k = 0; k < N; ++k) du[k] = b.scale * raw_at(rg, k) * dH[k];
            } else {
#pragma unroll
                for (int k = 0; k < N; ++k) du[k] = b.scale * dH[k];
            }
            if (!post) {
                if (live)
#pragma unroll
                    for (int k = 0; k < N; ++k) gt[k] = fmaf(b.scale * dH[k], raw_at(rx, k), gt[k]);
                if (g.dx && live) store_row<T, NT, C, VEC>(static_cast<T*>(g.dx) + i * b.ld_x, l, D, du);
                continue;
            }
            load_raw<float, NT, C, VEC>(b.post_w, l, D, rw);
            Raw<float, N, VEC> rb;
            if (LAYER && b.post_b) load_raw<float, NT, C, VEC>(b.post_b, l, D, rb);
            float s[2] = {0.f, 0.f};
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const float xh = elem<NT, VEC>(l, k) < D ? (raw_at(rx, k) - st.x) * st.y : 0.f;
                const float p = du[k] * raw_at(rw, k);
                s[0] = fmaf(p, xh, s[0]);
                if (LAYER) s[1] += p;
                if (live) {
                    float u = xh * raw_at(rw, k);
                    if (LAYER && b.post_b) u += raw_at(rb, k);
                    gt[k] = fmaf(b.scale * dH[k], u, gt[k]);
                    qw[k] = fmaf(du[k], xh, qw[k]);
                    if (LAYER) qb[k] += du[k];
                }
            }
            if (!g.dx) continue;   // (the same in every thread)
            row_sum<NT, 2>(s, red, slot);
            const float c1 = s[0] * inv_d, c0 = LAYER ? s[1] * inv_d : 0.f;
#pragma unroll
            for (int k = 0; k < N; ++k)
                du[k] = st.y * (du[k] * raw_at(rw, k) - c0 - (raw_at(rx, k) - st.x) * st.y * c1);
            if (live) store_row<T, NT, C, VEC>(static_cast<T*>(g.dx) + i * b.ld_x, l, D, du);
        }
        if (g.gate && b.gate_rows && q.pieces == 1) {   // the whole group was here
            combine(gt);
            if (rs == 0)
                store_row<float, NT, C, VEC>(g.gate + (base / b.gate_rows) * D, l, D, gt);
#pragma unroll
            for (int k = 0; k < N; ++k) gt[k] = 0.f;
        }
    }
    float* out = part + (long long)blockIdx.x * kPlanes * D;
    auto put = [&](bool wanted, int plane, float (&v)[N]) {
        if (!wanted) return;
        combine(v);
        if (rs == 0) store_row<float, NT, C, VEC>(out + (long long)plane * D, l, D, v);
    };
    put(g.pre_w, PL_PRE_W, pw);
    put(g.post_w, PL_POST_W, qw);
    put(g.gate && !(b.gate_rows && q.pieces == 1), PL_GATE, gt);
    if constexpr (LAYER) {
        put(g.pre_b, PL_PRE_B, pb);
        put(g.post_b, PL_POST_B, qb);
    }
}

// The blocks' partial sums of one plane and shard (gate of a group: of the group's pieces), 64
// columns to a block; its sixteen waves take runs of the blocks, joined in order.
__global__ __launch_bounds__(1024) void norm_join_kernel(BlockNormGrads g, NormDeal q, int R, int D,
                                                         bool group_gate,
                                                         const float* __restrict__ part)
{
    __shared__ float sum[16][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int d = blockIdx.y * 64 + lane;
    long long o = blockIdx.x;   // which output row: shards x planes, then the groups' gates
    int plane;
    long long first, n;
    float* out;
    if (o < (long long)R * kPlanes) {
        plane = (int)(o / R);
        o %= R;
        float* const outs[kPlanes] = {g.pre_w, g.post_w, group_gate ? nullptr : g.gate, g.pre_b, g.post_b};
        out = outs[plane];
        if (!out) return;
        out += o * g.ld;
        first = o * q.blocks_shard;
        n = q.blocks_shard;
    } else {
        o -= (long long)R * kPlanes;
        plane = PL_GATE;
        out = g.gate + o * D;
        first = o * q.pieces;
        n = q.pieces;
    }
    const long long per = (n + 15) / 16, b0 = w * per, b1 = min(n, b0 + per);
    float v = 0.f;
    if (d < D) {
        const float* p = part + (first * kPlanes + plane) * D + d;
#pragma unroll 4
        for (long long k = b0; k < b1; ++k) v += p[k * kPlanes * D];
    }
    sum[w][lane] = v;
    __syncthreads();
    if (w || d >= D) return;
#pragma unroll
    for (int k = 1; k < 16; ++k) v += sum[k][lane];
    out[d] = v;
}

size_t block_norm_bwd_bytes(const BlockNorm& b, int R)
{
    return std::max<size_t>(256, (size_t)norm_deal(b, R).blocks * kPlanes * b.D * 4);
}

template <typename T, int NT, int C>
static void launch_bwd(const BlockNorm& b, bool vec, const BlockNormGrads& g, const NormDeal& q,
                       float* part, hipStream_t s)
{
    const dim3 grid((unsigned)q.blocks), block(block_of(NT));
    if (vec && b.layer)
        hipLaunchKernelGGL((norm_bwd_kernel<T, NT, C, true, true>), grid, block, 0, s, b, g, q, part);
    else if (vec)
        hipLaunchKernelGGL((norm_bwd_kernel<T, NT, C, true, false>), grid, block, 0, s, b, g, q, part);
    else if (b.layer)
        hipLaunchKernelGGL((norm_bwd_kernel<T, NT, C, false, true>), grid, block, 0, s, b, g, q, part);
    else
        hipLaunchKernelGGL((norm_bwd_kernel<T, NT, C, false, false>), grid, block, 0, s, b, g, q, part);
}

hipError_t block_norm_bwd(const BlockNorm& b, int R, const BlockNormGrads& g, void* ws,
                          hipStream_t s)
{
    float* part = static_cast<float*>(ws);
    const NormDeal q = norm_deal(b, R);
    const bool group_gate = b.gate_rows != 0;
    if (q.blocks) {
        const bool vec = norm_vec(b, {g.h_out, g.x, g.dy, g.dh_out, g.dh, g.dx,
                                      group_gate ? g.gate : nullptr});
        auto go = [&](auto t) {
            using T = decltype(t);
            if (b.D <= 512) launch_bwd<T, 64, 1>(b, vec, g, q, part, s);
            else if (b.D <= 1024) launch_bwd<T, 128, 1>(b, vec, g, q, part, s);
            else if (b.D <= 2048) launch_bwd<T, 256, 1>(b, vec, g, q, part, s);
            else if (b.D <= 4096) launch_bwd<T, 512, 1>(b, vec, g, q, part, s);
            else if (b.D <= 8192) launch_bwd<T, 1024, 1>(b, vec, g, q, part, s);
            else launch_bwd<T, 1024, 2>(b, vec, g, q, part, s);
        };
        if (b.dt == DT_F32) go(float());
        else go(bf16_t());
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (!g.pre_w && !g.post_w && !g.gate && !g.pre_b && !g.post_b) return hipSuccess;
    const long long rows = (long long)R * kPlanes +
                           (group_gate && g.gate && q.pieces > 1 ? q.groups_shard * R : 0);
    hipLaunchKernelGGL(norm_join_kernel, dim3((unsigned)rows, (b.D + 63) / 64), dim3(1024), 0, s, g,
                       q, R, b.D, group_gate, part);
    return hipGetLastError();
}

}  // namespace mtx
