// The end of a residual block and the norm before the next one, in one pass over the rows:
//   u = norm(x) post_w + post_b (or x);  H = h + scale gate u;  y = norm(H) pre_w + pre_b
// with RMS or layer norm over the D elements of a row, and its gradients.  With H^ = (H - mean) r,
//   dH = dh_out + r (dy pre_w - [mean(dy pre_w)] - H^ mean(dy pre_w H^))     ([]: layer norm)
//   dh = dH;  du = scale gate dH;  dx likewise through x^ = (x - mean) r
//   d_pre_w = sum dy H^, d_pre_b = sum dy, d_post_w = sum du x^, d_post_b = sum du,
//   d_gate = scale sum dH u.
// Statistics and sums are fp32; only h_out, y, dh and dx are rounded to the tensors' type.
//
// A row is held in the registers of NT threads, C times 16 bytes each, so that every tensor is read
// and written once: both passes are bound by HBM.  Rows of at most 64 runs of elements take a wave,
// of at most 16 or 32 a quarter or half of one, and need no barrier.
#include "device_common.h"
#include "internal.h"

#include <algorithm>
#include <initializer_list>
#include <type_traits>

namespace mtx {

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// A thread's N = W C elements.  AL (rows of a multiple of W elements, aligned): runs of W, element k at
// ((k / W) NT + l) W + k % W, so that a wave's vector loads are contiguous.  Else singly, element
// k at k NT + l (unaligned vectors were slower: 8850 rows of 771 fp32, backward, 65 -> 89 us).
template <int NT, int W, bool AL> __device__ __forceinline__ int elem(int l, int k)
{
    return AL ? ((k / W) * NT + l) * W + k % W : k * NT + l;
}

// N elements as they are stored: 32-bit words (AL), or one by one.
template <typename T, int N, bool AL> struct Raw {
    unsigned w[AL ? N * (int)sizeof(T) / 4 : 1];
    T e[AL ? 1 : N];
};

// A row as a buffer of D elements: what lies past its end reads as zero and is not written, without a
// branch or a mask for it (8850 rows of 771 fp32, backward: 53 -> 47 us).  The pointer is the same
// in every lane of a wave.  Where a wave holds several rows (NT < 64), each lane adds its row's
// distance `off` (elements) from the wave's first, and names a place past any buffer for what its
// row does not have.
template <typename T, int NT>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t row_buffer(const T* p, int D)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(p), 0,
                                             NT < 64 ? 0x7fffffff : D * (int)sizeof(T), 0x00020000);
}

template <typename T, int NT> __device__ __forceinline__ int row_byte(int d, int off, int D)
{
    if (NT >= 64) return d * (int)sizeof(T);
    return d < D ? (off + d) * (int)sizeof(T) : (int)0x80000000;
}

template <typename T, int NT, int W, int C, bool AL>
__device__ __forceinline__ void load_raw(const T* p, int l, int D, Raw<T, W * C, AL>& o, int off = 0)
{
    const __amdgpu_buffer_rsrc_t r = row_buffer<T, NT>(p, D);
    if constexpr (AL) {
        constexpr int bytes = W * (int)sizeof(T);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int at = row_byte<T, NT>((c * NT + l) * W, off, D);
            if constexpr (bytes == 8) {
                const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(r, at, 0, 0);
                o.w[2 * c] = v[0];
                o.w[2 * c + 1] = v[1];
            } else {
#pragma unroll
                for (int q = 0; q < bytes / 16; ++q) {
                    const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(r, at + 16 * q, 0, 0);
#pragma unroll
                    for (int j = 0; j < 4; ++j) o.w[(c * (bytes / 16) + q) * 4 + j] = v[j];
                }
            }
        }
    } else {
#pragma unroll
        for (int k = 0; k < W * C; ++k) {
            const int at = row_byte<T, NT>(k * NT + l, off, D);
            if constexpr (sizeof(T) == 4)
                o.e[k] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(r, at, 0, 0));
            else
                o.e[k] = __builtin_amdgcn_raw_buffer_load_b16(r, at, 0, 0);
        }
    }
}

template <typename T, int N, bool AL>
__device__ __forceinline__ float raw_at(const Raw<T, N, AL>& o, int k)
{
    if constexpr (!AL) return to_f32<T>(o.e[k]);
    else if constexpr (sizeof(T) == 4) return __uint_as_float(o.w[k]);
    else return __uint_as_float(k % 2 ? o.w[k / 2] & 0xffff0000u : o.w[k / 2] << 16);
}

template <typename T, int NT, int W, int C, bool AL>
__device__ __forceinline__ void store_row(T* p, int l, int D, const float (&v)[W * C], int off = 0)
{
    const __amdgpu_buffer_rsrc_t r = row_buffer<T, NT>(p, D);
    if constexpr (AL) {
        constexpr int bytes = W * (int)sizeof(T);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int at = row_byte<T, NT>((c * NT + l) * W, off, D);
            T e[W];
#pragma unroll
            for (int k = 0; k < W; ++k) e[k] = from_f32<T>(v[W * c + k]);
            if constexpr (bytes == 8) {
                u32x2 raw;
                __builtin_memcpy(&raw, e, 8);
                __builtin_amdgcn_raw_buffer_store_b64(raw, r, at, 0, 0);
            } else {
#pragma unroll
                for (int q = 0; q < bytes / 16; ++q) {
                    u32x4 raw;
                    __builtin_memcpy(&raw, e + q * 16 / (int)sizeof(T), 16);
                    __builtin_amdgcn_raw_buffer_store_b128(raw, r, at + 16 * q, 0, 0);
                }
            }
        }
    } else {
#pragma unroll
        for (int k = 0; k < W * C; ++k) {
            const int at = row_byte<T, NT>(k * NT + l, off, D);
            const T e = from_f32<T>(v[k]);
            if constexpr (sizeof(T) == 4)
                __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, e), r, at, 0, 0);
            else
                __builtin_amdgcn_raw_buffer_store_b16(e, r, at, 0, 0);
        }
    }
}

// Sums over the NT threads of a row, the same bits in each.  `slot` alternates between calls: a
// wave writes the slot of two calls ago only after a barrier that follows all its reads.
template <int NT, int M>
__device__ __forceinline__ void row_sum(float (&v)[M], float (&red)[2][M][16], int& slot)
{
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int o = (NT < 64 ? NT : 64) / 2; o; o >>= 1) v[m] += __shfl_xor(v[m], o);
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
constexpr int bwd_block(int NT) { return NT < 512 ? 512 : NT; }

// A block holds block_of(NT) / NT rows at a time, one to a slot.  first: the wave's first slot (the same
// in all its lanes); sub: the lane's slot after it.
struct Slot {
    int first, sub;
};
template <int NT> __device__ __forceinline__ Slot row_slot()
{
    if (NT >= 64) return Slot{__builtin_amdgcn_readfirstlane(threadIdx.x / NT), 0};
    return Slot{__builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * (64 / NT),
                (int)(threadIdx.x & 63) / NT};
}

template <typename T, int W, int NT, int C, bool AL, bool LAYER>
__global__ __launch_bounds__(block_of(NT)) void norm_fwd_kernel(BlockNorm b, const T* h, const T* x,
                                                                T* h_out, T* y, float* stats,
                                                                long long row0)
{
    constexpr int N = W * C, RPB = block_of(NT) / NT;
    __shared__ float red[2][1][16];
    int slot = 0;
    const int l = threadIdx.x % NT, D = b.D;
    const float inv_d = 1.0f / (float)D;
    // (a block's rows run together: one past the end is as wide as nothing, read and written)
    const Slot sl = row_slot<NT>();
    const long long iw = row0 + (long long)blockIdx.x * RPB + sl.first, i = iw + sl.sub;
    const bool live = i < b.rows;
    const int Dl = live ? D : 0;
    const int oh = sl.sub * (int)b.ld_h, ox = sl.sub * (int)b.ld_x, oy = sl.sub * (int)b.ld_y;
    Raw<T, N, AL> rh, rx;
    load_raw<T, NT, W, C, AL>(h + iw * b.ld_h, l, Dl, rh, oh);
    if (x) load_raw<T, NT, W, C, AL>(x + iw * b.ld_x, l, Dl, rx, ox);
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
            const float t = LAYER && elem<NT, W, AL>(l, k) >= D ? 0.f : v[k] - mean;
            s[0] = fmaf(t, t, s[0]);
        }
        row_sum<NT, 1>(s, red, slot);
        const float r = 1.0f / sqrtf(s[0] * inv_d + b.eps);
        if (stats && live && l == 0)
            *reinterpret_cast<float2*>(stats + 4 * i + stat) = make_float2(mean, r);
        Raw<float, N, AL> rw, rb;
        load_raw<float, NT, W, C, AL>(w, l, D, rw);
        if (LAYER && bias) load_raw<float, NT, W, C, AL>(bias, l, D, rb);
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
            Raw<float, N, AL> rg;
            const long long gw = b.gate_rows ? iw / b.gate_rows : 0;
            const int og = NT < 64 && b.gate_rows ? (int)(i / b.gate_rows - gw) * D : 0;
            load_raw<float, NT, W, C, AL>(b.gate + gw * D, l, Dl, rg, og);
#pragma unroll
            for (int k = 0; k < N; ++k) H[k] = fmaf(b.scale * raw_at(rg, k), u[k], H[k]);
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) H[k] = fmaf(b.scale, u[k], H[k]);
        }
        if (h_out) store_row<T, NT, W, C, AL>(h_out + iw * b.ld_h, l, Dl, H, oh);
    }
    if (!y) return;
    norm(H, b.pre_w, b.pre_b, 2);
    store_row<T, NT, W, C, AL>(y + iw * b.ld_y, l, Dl, H, oy);
}

static bool al16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Elements of a run: 16 bytes; four where they are loaded singly.
template <typename T, bool AL> constexpr int kRun = sizeof(T) == 4 || !AL ? 4 : 8;

// Calls go(type, layer norm, aligned) as constants.
template <class F> static void with_form(const BlockNorm& b, bool al, F go)
{
    auto by_type = [&](auto t) {
        if (b.layer) al ? go(t, std::true_type(), std::true_type()) : go(t, std::true_type(), std::false_type());
        else al ? go(t, std::false_type(), std::true_type()) : go(t, std::false_type(), std::false_type());
    };
    if (b.dt == DT_F32) by_type(float());
    else by_type(bf16_t());
}

static bool norm_vec(const BlockNorm& b, std::initializer_list<const void*> ptrs)
{
    const int w = b.dt == DT_F32 ? 4 : 8;
    bool ok = b.D % w == 0 && b.ld_h % w == 0 && b.ld_x % w == 0 && b.ld_y % w == 0 &&
              al16(b.post_w) && al16(b.post_b) && al16(b.gate) && al16(b.pre_w) && al16(b.pre_b);
    for (const void* p : ptrs) ok = ok && al16(p);
    return ok;
}

// Threads of a row of D elements in runs of w (C = 1 up to 1024).  Rows that share a wave must lie within
// the reach of its 31-bit distances: `far` is the largest one, in bytes.
static int row_threads(int D, int w, double far)
{
    int nt = far < 2147483647.0 ? 16 : 64;
    while (nt < 1024 && nt * w < D) nt *= 2;
    return nt;
}

// Calls f(NT, C) as constants.
template <int W, class F> static void with_row_shape(int D, int nt, F f)
{
    const std::integral_constant<int, 1> one;
    if (nt == 16) f(std::integral_constant<int, 16>(), one);
    else if (nt == 32) f(std::integral_constant<int, 32>(), one);
    else if (nt == 64) f(std::integral_constant<int, 64>(), one);
    else if (nt == 128) f(std::integral_constant<int, 128>(), one);
    else if (nt == 256) f(std::integral_constant<int, 256>(), one);
    else if (nt == 512) f(std::integral_constant<int, 512>(), one);
    else if (D <= 1024 * W) f(std::integral_constant<int, 1024>(), one);
    else if (D <= 2048 * W) f(std::integral_constant<int, 1024>(), std::integral_constant<int, 2>());
    else f(std::integral_constant<int, 1024>(), std::integral_constant<int, W == 8 ? 2 : 4>());
}

// Largest distance in bytes of a tensor's rows that share a wave and lie `step` rows apart.
static double wave_reach(const BlockNorm& b, long long step)
{
    const double ld = (double)std::max({b.ld_h, b.ld_x, b.ld_y});
    return (3.0 * step + 1.0) * ld * (b.dt == DT_F32 ? 4 : 2);
}

hipError_t block_norm_fwd(const BlockNorm& b, const void* h, const void* x, void* h_out, void* y,
                          float* stats, hipStream_t s)
{
    if (b.rows == 0) return hipSuccess;
    const bool al = norm_vec(b, {h, x, h_out, y});
    auto go = [&](auto t, auto layer, auto aligned) {
        using T = decltype(t);
        constexpr bool LAYER = decltype(layer)::value, AL = decltype(aligned)::value;
        constexpr int W = kRun<T, AL>;
        with_row_shape<W>(b.D, row_threads(b.D, W, wave_reach(b, 1)), [&](auto nt, auto c) {
            constexpr int NT = decltype(nt)::value, C = decltype(c)::value;
            constexpr int RPB = block_of(NT) / NT;
            // (a launch has at most 2^32 threads)
            constexpr long long most = 1LL << 21;
            for (long long r = 0; r < b.rows; r += most * RPB) {
                const long long n = std::min(most, (b.rows - r + RPB - 1) / RPB);
                hipLaunchKernelGGL((norm_fwd_kernel<T, W, NT, C, AL, LAYER>), dim3((unsigned)n),
                                   dim3(block_of(NT)), 0, s, b, static_cast<const T*>(h),
                                   static_cast<const T*>(x), static_cast<T*>(h_out),
                                   static_cast<T*>(y), stats, r);
            }
        });
    };
    with_form(b, al, go);
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
    int pieces, chunk, gpb, Dp;      // Dp: D to a multiple of 4, the partial sums' rows
    int threads, run;                // of a row; elements of a thread's run
    long long blocks_shard, blocks;
};

static NormDeal norm_deal_runs(const BlockNorm& b, int R, int w)
{
    NormDeal q{};
    q.run = w;
    const long long nb = b.rows / R;
    q.Dp = (b.D + 3) / 4 * 4;
    q.group = b.gate_rows ? b.gate_rows : nb;
    q.groups_shard = q.group ? nb / q.group : 0;
    // (rows that share a wave: neighbours, or of neighbouring gate groups)
    q.threads = row_threads(b.D, w, wave_reach(b, b.gate_rows ? b.gate_rows : 1));
    const int slots_block = q.threads < 512 ? 512 / q.threads : 1;
    // At most the blocks that 256 compute units hold at 16 waves each (the kernels' registers):
    // one more would run alone.  Fewer rows to a block than that gives only cost partial sums.
    const long long slots = 256LL * 1024 / std::max(512, q.threads);
    for (long long rows = std::max<long long>(1, nb * R / slots);; rows += std::max<long long>(1, rows / 16)) {
        q.gpb = q.pieces = 1;
        q.chunk = (int)q.group;
        if (q.group > rows) {
            q.pieces = (int)((q.group + rows - 1) / rows);
            q.chunk = (int)((q.group + q.pieces - 1) / q.pieces);
        } else if (q.group && q.groups_shard > 1) {
            // several groups, one to a slot at a time; fewer than slots: a block for each
            const long long g = rows / q.group / slots_block * slots_block;
            q.gpb = (int)std::max<long long>(1, std::min(g, q.groups_shard));
        }
        q.blocks_shard = q.pieces > 1 ? q.groups_shard * q.pieces : (q.groups_shard + q.gpb - 1) / q.gpb;
        if (q.blocks_shard * R <= slots || rows >= nb) break;
    }
    q.blocks = q.blocks_shard * R;
    return q;
}

// A block of several groups with the biases' sums has no registers for runs of 8 (65536 x 128 bf16, gates
// of 2 rows: 73 us, with runs of 4 44; a block of one group: 32768 x 512 54 and 72).
static NormDeal norm_deal(const BlockNorm& b, int R, bool al)
{
    const NormDeal q = norm_deal_runs(b, R, b.dt == DT_F32 || !al ? 4 : 8);
    return q.run == 8 && q.gpb > 1 && b.layer ? norm_deal_runs(b, R, 4) : q;
}

// planes of a block's partial sums
enum { PL_PRE_W, PL_POST_W, PL_GATE, PL_PRE_B, PL_POST_B, kPlanes };

// Within a group du = scale gate dH with one gate vector, so the sums over its rows come from two:
//   t1 = sum dH x^ (x where there is no post norm),  t0 = sum dH:
//   d_post_w = scale gate t1, d_post_b = scale gate t0, d_gate = scale (post_w t1 + post_b t0).
// MANY: a block of several whole groups adds d_post_w and d_post_b over them.  The next row's dy and
// h_out are loaded while a row is worked on; dh_out and x arrive during its first sum (8850 x 771:
// 47 -> 44 us).  8192 x 4096 bf16, four shards: 97 us, 4.4 TB/s with the partial sums; half the
// blocks 128, twice as many 100.
template <typename T, int W, int NT, int C, bool AL, bool LAYER, bool MANY>
__global__ __launch_bounds__(bwd_block(NT), C == 1 ? 4 : 1) void norm_bwd_kernel(BlockNorm b, BlockNormGrads g,
                                                                NormDeal q, float* __restrict__ part)
{
    constexpr int N = W * C, RPB = bwd_block(NT) / NT, M = LAYER ? 2 : 1;
    __shared__ float red[2][M][16];
    __shared__ float comb[RPB > 1 ? RPB - 1 : 1][RPB > 1 ? N * NT : 1];
    int slot = 0;
    const int l = threadIdx.x % NT, D = b.D;
    const Slot sl = row_slot<NT>();
    const int rs = sl.first + sl.sub;
    const float inv_d = 1.0f / (float)D;
    const long long shard = blockIdx.x / q.blocks_shard, bs = blockIdx.x % q.blocks_shard;
    const long long nb = q.group * q.groups_shard;
    // MANY: groups g0 .. g1 - 1 of the shard, one to a slot at a time.  Else a run of the rows of group g0
    // (interleaved rows took the same time), one to a slot.
    const long long g0 = MANY ? bs * q.gpb : bs / q.pieces;
    const long long g1 = MANY ? min(g0 + q.gpb, q.groups_shard) : q.groups_shard;
    // (one group is a loop as well: with the compiler seeing a single pass, 8850 x 771 fp32 took 48 us, so 44)
    const long long gstep = MANY ? RPB : q.groups_shard;
    const int first = MANY ? 0 : (int)(bs % q.pieces) * q.chunk;
    const int rows = MANY ? (int)q.group : (int)max(0LL, min((long long)q.chunk, q.group - first));
    constexpr int rstep = MANY ? 1 : RPB;
    // distance of a lane's rows from the first of its wave
    const long long apart = MANY ? q.group : 1;
    const int oh = sl.sub * (int)(apart * b.ld_h), ox = sl.sub * (int)(apart * b.ld_x),
              oy = sl.sub * (int)(apart * b.ld_y), og = MANY && b.gate_rows ? sl.sub * D : 0;
    const bool has_x = g.x != nullptr, has_y = g.dy != nullptr;
    const bool post = b.post_w != nullptr;
    float pw[N], t1[N], pb[LAYER ? N : 1], t0[LAYER ? N : 1];
    float qw[MANY ? N : 1], qb[MANY && LAYER ? N : 1];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        pw[k] = t1[k] = 0.f;
        if (LAYER) pb[k] = t0[k] = 0.f;
        if (MANY) qw[k] = 0.f;
        if (MANY && LAYER) qb[k] = 0.f;
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
    float* out = part + (long long)blockIdx.x * kPlanes * q.Dp;
    auto put = [&](int plane, const float (&v)[N]) {
        if (rs == 0) store_row<float, NT, W, C, AL>(out + (long long)plane * q.Dp, l, D, v);
    };
    // the first row of the wave; a slot past the rows (the groups) is as wide as nothing
    auto row_of = [&](long long gi, int j) {
        return shard * nb + (MANY ? (gi + sl.first) * q.group + j
                                  : gi * q.group + first + j + sl.first);
    };
    auto width = [&](long long gi, int j) {
        return (MANY ? gi + rs < g1 : j + rs < rows) ? D : 0;
    };
    Raw<T, N, AL> rH, ry;
    auto load_y = [&](long long gi, int j) {
        const long long i = row_of(gi, j);
        const int Dl = width(gi, j);
        load_raw<T, NT, W, C, AL>(static_cast<const T*>(g.dy) + i * b.ld_y, l, Dl, ry, oy);
        load_raw<T, NT, W, C, AL>(static_cast<const T*>(g.h_out) + i * b.ld_h, l, Dl, rH, oh);
    };
    if (has_y && rows && g0 < g1) load_y(g0, 0);
    for (long long gi = g0; gi < g1; gi += gstep) {
        // (the wave's first group)
        const long long gate_row = b.gate_rows ? shard * q.groups_shard + gi + (MANY ? sl.first : 0) : 0;
        const float* gate = b.gate ? b.gate + gate_row * D : nullptr;
        const bool live_group = !MANY || gi + rs < g1;
        for (int j0 = 0; j0 < rows; j0 += rstep) {
            const long long i = row_of(gi, j0);
            const int Dl = width(gi, j0);
            const bool live = Dl != 0;
            Raw<T, N, AL> ro, rx;
            Raw<float, N, AL> rw;
            float4 st = make_float4(0.f, 0.f, 0.f, 0.f);
            if (g.stats && live)
                st = *reinterpret_cast<const float4*>(g.stats + 4 * (i + sl.sub * apart));
            if (g.dh_out)
                load_raw<T, NT, W, C, AL>(static_cast<const T*>(g.dh_out) + i * b.ld_h, l, Dl, ro, oh);
            if (has_x) load_raw<T, NT, W, C, AL>(static_cast<const T*>(g.x) + i * b.ld_x, l, Dl, rx, ox);
            // the row's loads are issued here, not moved behind the sums
            __builtin_amdgcn_sched_barrier(0);
            float dH[N];
            if (has_y) {
                load_raw<float, NT, W, C, AL>(b.pre_w, l, D, rw);
                float s[M] = {};
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    const float p = raw_at(ry, k) * raw_at(rw, k);
                    s[0] = fmaf(p, (raw_at(rH, k) - st.z) * st.w, s[0]);
                    if (LAYER) s[M - 1] += p;
                }
                row_sum<NT, M>(s, red, slot);
                const float c1 = s[0] * inv_d, c0 = LAYER ? s[M - 1] * inv_d : 0.f;
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    const float dy = raw_at(ry, k), hat = (raw_at(rH, k) - st.z) * st.w;
                    dH[k] = (g.dh_out ? raw_at(ro, k) : 0.f) +
                            st.w * (dy * raw_at(rw, k) - c0 - hat * c1);
                    if (live) {
                        pw[k] = fmaf(dy, hat, pw[k]);
                        if (LAYER) pb[k] += dy;
                    }
                }
            } else {
#pragma unroll
                for (int k = 0; k < N; ++k) dH[k] = raw_at(ro, k);
            }
            if (g.dh) {
                if (g.relu_h) {
                    float v[N];
#pragma unroll
                    for (int k = 0; k < N; ++k) v[k] = raw_at(rH, k) > 0.f ? dH[k] : 0.f;
                    store_row<T, NT, W, C, AL>(static_cast<T*>(g.dh) + i * b.ld_h, l, Dl, v, oh);
                } else {
                    store_row<T, NT, W, C, AL>(static_cast<T*>(g.dh) + i * b.ld_h, l, Dl, dH, oh);
                }
            }
            if (has_y) {
                if (j0 + rstep < rows) load_y(gi, j0 + rstep);
                else if (MANY && gi + gstep < g1) load_y(gi + gstep, 0);
            }
            if (!has_x) continue;
            if (live) {
                // (past D, dH is not 0; its sums there are not stored)
                const float m = post ? st.x : 0.f, r = post ? st.y : 1.f;
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    t1[k] = fmaf(dH[k], (raw_at(rx, k) - m) * r, t1[k]);
                    if (LAYER) t0[k] += dH[k];
                }
            }
            if (!g.dx) continue;   // (the same in every thread)
            // dH becomes du = scale gate dH, then dx
            if (gate) {
                Raw<float, N, AL> rg;
                load_raw<float, NT, W, C, AL>(gate, l, Dl, rg, og);
#pragma unroll
                for (int k = 0; k < N; ++k) dH[k] *= b.scale * raw_at(rg, k);
            } else {
#pragma unroll
                for (int k = 0; k < N; ++k) dH[k] *= b.scale;
            }
            if (post) {
                load_raw<float, NT, W, C, AL>(b.post_w, l, D, rw);
                float s[M] = {};
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    dH[k] *= raw_at(rw, k);   // (0 past D)
                    s[0] = fmaf(dH[k], (raw_at(rx, k) - st.x) * st.y, s[0]);
                    if (LAYER) s[M - 1] += dH[k];
                }
                row_sum<NT, M>(s, red, slot);
                const float c1 = s[0] * inv_d, c0 = LAYER ? s[M - 1] * inv_d : 0.f;
#pragma unroll
                for (int k = 0; k < N; ++k)
                    dH[k] = st.y * (dH[k] - c0 - (raw_at(rx, k) - st.x) * st.y * c1);
            }
            store_row<T, NT, W, C, AL>(static_cast<T*>(g.dx) + i * b.ld_x, l, Dl, dH, ox);
        }
        // the group's sums on x's side
        if (!g.gate && !g.post_w && !g.post_b) continue;
        if constexpr (!MANY) {
            combine(t1);
            if constexpr (LAYER) combine(t0);
        }
        float v[N];
        if (g.gate) {
            Raw<float, N, AL> rw, rb;
            if (post) load_raw<float, NT, W, C, AL>(b.post_w, l, D, rw);
            if (LAYER && b.post_b) load_raw<float, NT, W, C, AL>(b.post_b, l, D, rb);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                v[k] = post ? raw_at(rw, k) * t1[k] : t1[k];
                if constexpr (LAYER)
                    if (b.post_b) v[k] = fmaf(raw_at(rb, k), t0[k], v[k]);
                v[k] *= b.scale;
            }
            if (MANY || (b.gate_rows && q.pieces == 1)) {   // the whole group was here
                store_row<float, NT, W, C, AL>(g.gate + gate_row * D, l,
                                               MANY ? (live_group ? D : 0) : rs ? 0 : D, v, og);
            } else {
                put(PL_GATE, v);
            }
        }
        if (g.post_w || g.post_b) {
            Raw<float, N, AL> rg;
            if (gate) load_raw<float, NT, W, C, AL>(gate, l, live_group ? D : 0, rg, og);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const float f = gate ? b.scale * raw_at(rg, k) : b.scale;
                t1[k] *= f;
                if constexpr (LAYER) t0[k] *= f;
                if constexpr (MANY) {
                    qw[k] += t1[k];
                    if constexpr (LAYER) qb[k] += t0[k];
                }
            }
        }
        if constexpr (MANY) {
#pragma unroll
            for (int k = 0; k < N; ++k) {
                t1[k] = 0.f;
                if constexpr (LAYER) t0[k] = 0.f;
            }
        }
    }
    if (g.pre_w) {
        combine(pw);
        put(PL_PRE_W, pw);
    }
    if constexpr (MANY) {
        if (g.post_w) {
            combine(qw);
            put(PL_POST_W, qw);
        }
    } else {
        if (g.post_w) put(PL_POST_W, t1);
    }
    if constexpr (LAYER) {
        if (g.pre_b) {
            combine(pb);
            put(PL_PRE_B, pb);
        }
        if constexpr (MANY) {
            if (g.post_b) {
                combine(qb);
                put(PL_POST_B, qb);
            }
        } else {
            if (g.post_b) put(PL_POST_B, t0);
        }
    }
}

// The blocks' partial sums of one plane and shard (gate of a group: of the group's pieces), 256
// columns to a block; its sixteen waves take runs of the partial sums, joined in order.
__global__ __launch_bounds__(1024) void norm_join_kernel(BlockNormGrads g, NormDeal q, int R, int D,
                                                         bool group_gate,
                                                         const float* __restrict__ part)
{
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    __shared__ f32x4 sum[16][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int d = blockIdx.y * 256 + lane * 4;
    long long o = blockIdx.x;   // which output row: shards x planes, then the groups' gates
    int plane;
    long long first, n;
    float* out;
    if (o < (long long)R * kPlanes) {
        plane = (int)(o / R);
        o %= R;
        out = plane == PL_PRE_W ? g.pre_w : plane == PL_POST_W ? g.post_w : plane == PL_PRE_B ? g.pre_b
              : plane == PL_POST_B ? g.post_b : group_gate ? nullptr : g.gate;
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
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (d < D) {
        const f32x4* p = reinterpret_cast<const f32x4*>(part + (first * kPlanes + plane) * q.Dp + d);
        const long long step = kPlanes * (q.Dp / 4);
        long long k = b0;
        for (; k + 4 <= b1; k += 4) {
            f32x4 t[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) t[j] = p[(k + j) * step];
#pragma unroll
            for (int j = 0; j < 4; ++j) v += t[j];
        }
        for (; k < b1; ++k) v += p[k * step];
    }
    sum[w][lane] = v;
    __syncthreads();
    if (w || d >= D) return;
#pragma unroll
    for (int k = 1; k < 16; ++k) v += sum[k][lane];
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (d + k < D) out[d + k] = v[k];
}

size_t block_norm_bwd_bytes(const BlockNorm& b, int R)
{
    const NormDeal q = norm_deal(b, R, true), u = norm_deal(b, R, false);
    return std::max<size_t>(256, (size_t)std::max(q.blocks, u.blocks) * kPlanes * q.Dp * 4);
}

hipError_t block_norm_bwd(const BlockNorm& b, int R, const BlockNormGrads& g, void* ws,
                          hipStream_t s)
{
    float* part = static_cast<float*>(ws);
    const bool group_gate = b.gate_rows != 0;
    const bool al = norm_vec(b, {g.h_out, g.x, g.dy, g.dh_out, g.dh, g.dx,
                                 group_gate ? g.gate : nullptr});
    const NormDeal q = norm_deal(b, R, al);
    if (q.blocks) {
        auto go = [&](auto t, auto layer, auto aligned) {
            using T = decltype(t);
            constexpr bool LAYER = decltype(layer)::value, AL = decltype(aligned)::value;
            auto launch = [&](auto w, auto many) {
                constexpr int W = decltype(w)::value;
                constexpr bool MANY = decltype(many)::value;
                with_row_shape<W>(b.D, q.threads, [&](auto nt, auto c) {
                    constexpr int NT = decltype(nt)::value, C = decltype(c)::value;
                    hipLaunchKernelGGL((norm_bwd_kernel<T, W, NT, C, AL, LAYER, MANY>),
                                       dim3((unsigned)q.blocks), dim3(bwd_block(NT)), 0, s, b, g, q,
                                       part);
                });
            };
            const std::integral_constant<int, kRun<T, AL>> full;
            if constexpr (kRun<T, AL> == 8 && LAYER) {
                if (q.gpb > 1) launch(std::integral_constant<int, 4>(), std::true_type());
                else launch(full, std::false_type());
            } else {
                if (q.gpb > 1) launch(full, std::true_type());
                else launch(full, std::false_type());
            }
        };
        with_form(b, al, go);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (!g.pre_w && !g.post_w && !g.gate && !g.pre_b && !g.post_b) return hipSuccess;
    const long long rows = (long long)R * kPlanes +
                           (group_gate && g.gate && q.pieces > 1 ? q.groups_shard * R : 0);
    if (q.blocks) timing_split(s, "join");
    hipLaunchKernelGGL(norm_join_kernel, dim3((unsigned)rows, (b.D + 255) / 256), dim3(1024), 0, s, g,
                       q, R, b.D, group_gate, part);
    return hipGetLastError();
}

}  // namespace mtx
