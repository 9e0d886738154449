// C ABI of the operators on caller tensors: token embedding, block norms, gradient clipping
// (include/mtx.h).  Arguments are checked here; the kernels are in embed.hip, blocknorm.hip and
// clip.hip.
#include "mtx.h"

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <utility>
#include <vector>

#include "api_common.h"
#include "internal.h"

using namespace mtx;

namespace {

bool known_type(int t) { return t == MTX_F32 || t == MTX_BF16; }
size_t type_size(int t) { return t == MTX_F32 ? 4 : 2; }

// A tensor's bytes: `rows` rows of `bytes` bytes, `stride` apart (at least `bytes`); bytes = 0 for an
// absent one.
struct Span {
    const void* p;
    size_t bytes;
    bool written;
    size_t rows = 1, stride = 0;
};

Span rows_span(const void* p, long long rows, long long D, long long ld, size_t es, bool written)
{
    return Span{p, p && rows > 0 ? (size_t)D * es : 0, written, (size_t)rows, (size_t)ld * es};
}

// Sum over 0 <= i < n of floor((a i + b) / m) for a, b >= 0 and m > 0: the lattice points under a
// line.  Whole multiples of m come out of a and b first; the rest is counted by rows (row k holds
// the i with a i + b >= k m), which is the same sum with a and m exchanged.
typedef __int128 wide;
wide points_under_line(wide n, wide a, wide b, wide m)
{
    if (n <= 0) return 0;
    const wide sum = a / m * (n * (n - 1) / 2) + b / m * n;
    a %= m;
    b %= m;
    const wide rows = (a * (n - 1) + b) / m;
    if (rows == 0) return sum;
    return sum + rows * n - points_under_line(rows, m, m - b + a - 1, a);
}

wide floor_div(wide x, wide m) { return x >= 0 ? x / m : -((-x + m - 1) / m); }

// Whether two tensors share a byte; the columns of one matrix may be several tensors.
bool share_bytes(const Span& a, const Span& b)
{
    if (!a.bytes || !b.bytes) return false;
    if (!overlap(a.p, (a.rows - 1) * a.stride + a.bytes, b.p, (b.rows - 1) * b.stride + b.bytes))
        return false;
    if (a.rows == 1 && b.rows == 1) return true;
    // Row i of a starts x = d + i sa behind b.  It meets the rows j of b with x - lb < j sb < x + la:
    // floor((x + la - 1) / sb) - floor((x - lb) / sb) of them, of which 0 <= j < b.rows leaves one
    // at least for the i of i0 .. i1, if it is not empty.
    const wide la = (wide)a.bytes, lb = (wide)b.bytes;
    const wide sa = a.rows > 1 ? (wide)a.stride : la, sb = b.rows > 1 ? (wide)b.stride : lb;
    const wide d = (wide)reinterpret_cast<uintptr_t>(a.p) - (wide)reinterpret_cast<uintptr_t>(b.p);
    const wide i0 = std::max<wide>(0, -floor_div(la - 1 + d, sa));
    const wide i1 = std::min<wide>((wide)a.rows - 1,
                                   floor_div(((wide)b.rows - 1) * sb + lb - 1 - d, sa));
    // (both floors of a multiple of sb more, so that nothing is negative)
    const wide x0 = d + i0 * sa + (la + lb + sb) / sb * sb;
    return points_under_line(i1 - i0 + 1, sa, x0 + la - 1, sb) >
           points_under_line(i1 - i0 + 1, sa, x0 - lb, sb);
}

// Whether a written tensor overlaps any other one.
template <class List> bool spans_overlap(const List& list)
{
    for (auto a = std::begin(list); a != std::end(list); ++a)
        for (auto b = a + 1; b != std::end(list); ++b)
            if ((a->written || b->written) && share_bytes(*a, *b)) return true;
    return false;
}

bool spans_overlap(std::initializer_list<Span> list) { return spans_overlap<>(list); }

constexpr size_t kMaxRows = 2147483647;
constexpr size_t kMaxTokens = (size_t)1 << 30;
constexpr int kMaxEmbedD = 1 << 24;

int check_embed(int V, int D, size_t n, int R)
{
    if (V < 1 || D < 1) return fail(MTX_EINVAL, "V and D must be >= 1 (got %d, %d)", V, D);
    if (D > kMaxEmbedD) return fail(MTX_EINVAL, "D must be at most %d (got %d)", kMaxEmbedD, D);
    if (R < 1 || R > 65536) return fail(MTX_EINVAL, "R must lie in 1 .. 65536 (got %d)", R);
    if (n > kMaxTokens || n * (size_t)R > kMaxTokens)
        return fail(MTX_EINVAL, "more than 2^30 tokens");
    if ((size_t)V * R > ((size_t)1 << 28)) return fail(MTX_EINVAL, "more than 2^28 table rows");
    if (n * (size_t)R * D > ((size_t)1 << 36)) return fail(MTX_EINVAL, "more than 2^36 elements");
    return MTX_OK;
}

}  // namespace

extern "C" {

int mtx_embed_forward(const void* w, int w_type, int V, int D, const int32_t* tokens, size_t n,
                      int pad, float scale, void* y, int y_type, size_t ldy, void* stream)
{
    const int rc = check_embed(V, D, n, 1);
    if (rc) return rc;
    if (!known_type(w_type) || !known_type(y_type))
        return fail(MTX_EINVAL, "w_type and y_type must be MTX_F32 or MTX_BF16");
    if (!std::isfinite(scale)) return fail(MTX_EINVAL, "scale must be finite");
    if (!w) return fail(MTX_EINVAL, "w must not be NULL");
    if (n == 0) return MTX_OK;
    if (!tokens || !y) return fail(MTX_EINVAL, "tokens and y must not be NULL");
    if (ldy < (size_t)D) return fail(MTX_EINVAL, "ldy must be >= D");
    const size_t ew = type_size(w_type), ey = type_size(y_type);
    if (ldy > ((size_t)1 << 62) / (n * ey)) return fail(MTX_EINVAL, "sizes overflow");
    if (!aligned(w, ew) || !aligned(y, ey) || !aligned(tokens, 4))
        return fail(MTX_EINVAL, "pointers must be aligned to their element size");
    if (spans_overlap({rows_span(y, n, D, ldy, ey, true), Span{w, (size_t)V * D * ew, false},
                       Span{tokens, n * 4, false}}))
        return fail(MTX_EINVAL, "y overlaps an input");
    HIP_TRY(embed_fwd(w, (Dt)w_type, V, D, tokens, (long long)n, pad, scale, y, (Dt)y_type,
                      (long long)ldy, static_cast<hipStream_t>(stream)), "mtx_embed_forward");
    return MTX_OK;
}

int mtx_embed_sizes(size_t n, int R, int V, int D, size_t* workspace_bytes)
{
    if (!workspace_bytes) return fail(MTX_EINVAL, "workspace_bytes is NULL");
    const int rc = check_embed(V, D, n, R);
    if (rc) return rc;
    *workspace_bytes = embed_bwd_bytes((long long)n, R, V, D);
    return MTX_OK;
}

int mtx_embed_backward(const int32_t* tokens, size_t n, int R, const void* dy, int dy_type,
                       size_t lddy, int V, int D, int pad, float scale, float* grads, size_t ld,
                       int accumulate, void* workspace, size_t workspace_bytes, void* stream)
{
    const int rc = check_embed(V, D, n, R);
    if (rc) return rc;
    if (!known_type(dy_type)) return fail(MTX_EINVAL, "dy_type must be MTX_F32 or MTX_BF16");
    if (!std::isfinite(scale)) return fail(MTX_EINVAL, "scale must be finite");
    if (!grads || (n && (!tokens || !dy)))
        return fail(MTX_EINVAL, "tokens, dy and grads must not be NULL");
    if (lddy < (size_t)D) return fail(MTX_EINVAL, "lddy must be >= D");
    const size_t vd = (size_t)V * D;
    if (ld < vd) return fail(MTX_EINVAL, "ld must be >= V * D");
    const size_t es = type_size(dy_type), N = n * R;
    if (ld > ((size_t)1 << 60) / R || (N && lddy > ((size_t)1 << 60) / N))
        return fail(MTX_EINVAL, "sizes overflow");
    if (!aligned(tokens, 4) || !aligned(grads, 4) || !aligned(dy, es))
        return fail(MTX_EINVAL, "pointers must be aligned to their element size");
    const size_t need = embed_bwd_bytes((long long)n, R, V, D);
    if (!workspace || !aligned(workspace, 16))
        return fail(MTX_EINVAL, "the workspace must be 16-byte aligned and not NULL");
    if (workspace_bytes < need)
        return fail(MTX_ENOMEM, "workspace too small: %zu bytes given, %zu needed",
                    workspace_bytes, need);
    if (spans_overlap({rows_span(grads, R, vd, ld, 4, true), Span{workspace, need, true},
                       rows_span(dy, N, D, lddy, es, false), Span{tokens, N * 4, false}}))
        return fail(MTX_EINVAL, "grads, dy, tokens and the workspace must not overlap");
    HIP_TRY(embed_bwd(tokens, (long long)n, R, dy, (Dt)dy_type, (long long)lddy, V, D, pad, scale,
                      grads, (long long)ld, accumulate != 0, workspace,
                      static_cast<hipStream_t>(stream)), "mtx_embed_backward");
    return MTX_OK;
}

}  // extern "C"

// The checks of a norm description that need no tensors; fills b with resolved strides.
static int check_norm(const mtx_norm_desc* d, BlockNorm& b)
{
    if (!d) return fail(MTX_EINVAL, "the description is NULL");
    if (d->kind != MTX_NORM_RMS && d->kind != MTX_NORM_LAYER)
        return fail(MTX_EINVAL, "unknown norm kind %d", d->kind);
    if (!known_type(d->dtype)) return fail(MTX_EINVAL, "dtype must be MTX_F32 or MTX_BF16");
    if (d->D < 1) return fail(MTX_EINVAL, "D must be >= 1 (got %d)", d->D);
    if (d->D > kNormMaxD)
        return fail(MTX_EUNSUPPORTED, "D must be at most %d (got %d)", kNormMaxD, d->D);
    if (d->rows > kMaxRows) return fail(MTX_EINVAL, "more than 2^31 - 1 rows");
    if (!std::isfinite(d->eps) || d->eps < 0.0f || !std::isfinite(d->scale))
        return fail(MTX_EINVAL, "eps must be finite and >= 0, scale finite");
    if (d->kind == MTX_NORM_RMS && (d->post_b || d->pre_b))
        return fail(MTX_EINVAL, "an RMS norm has no bias");
    if ((d->post_b && !d->post_w) || (d->pre_b && !d->pre_w))
        return fail(MTX_EINVAL, "a bias needs its weight");
    if (d->gate_rows && (!d->gate || d->rows % d->gate_rows))
        return fail(MTX_EINVAL, "gate_rows needs a gate, and must divide rows");
    for (const float* p : {d->post_w, d->post_b, d->gate, d->pre_w, d->pre_b})
        if (!aligned(p, 4)) return fail(MTX_EINVAL, "weights must be 4-byte aligned");
    size_t ld[3] = {d->ld_h, d->ld_x, d->ld_y};
    for (size_t& l : ld) {
        if (l == 0) l = (size_t)d->D;
        if (l < (size_t)d->D) return fail(MTX_EINVAL, "a row stride is below D");
        if (l > ((size_t)1 << 28)) return fail(MTX_EINVAL, "a row stride is above 2^28");
    }
    b.layer = d->kind == MTX_NORM_LAYER;
    b.dt = (Dt)d->dtype;
    b.rows = (long long)d->rows;
    b.D = d->D;
    b.eps = d->eps;
    b.scale = d->scale;
    b.gate_rows = (long long)d->gate_rows;
    b.post_w = d->post_w; b.post_b = d->post_b; b.gate = d->gate;
    b.pre_w = d->pre_w; b.pre_b = d->pre_b;
    b.ld_h = (long long)ld[0]; b.ld_x = (long long)ld[1]; b.ld_y = (long long)ld[2];
    return MTX_OK;
}

// Weights and gates are only read: spans of a description's.
#define NORM_PARAM_SPANS(b)                                                                     \
    Span{(b).post_w, (b).post_w ? (size_t)(b).D * 4 : 0, false},                                \
        Span{(b).post_b, (b).post_b ? (size_t)(b).D * 4 : 0, false},                            \
        Span{(b).pre_w, (b).pre_w ? (size_t)(b).D * 4 : 0, false},                              \
        Span{(b).pre_b, (b).pre_b ? (size_t)(b).D * 4 : 0, false},                              \
        Span{(b).gate, (b).gate ? (size_t)((b).gate_rows ? (b).rows / (b).gate_rows : 1) * (b).D * 4 : 0, false}

extern "C" {

int mtx_block_norm_forward(const mtx_norm_desc* d, const void* h, const void* x, void* h_out,
                           void* y, float* stats, void* stream)
{
    BlockNorm b{};
    const int rc = check_norm(d, b);
    if (rc) return rc;
    if (!x && (h_out || b.post_w || b.gate))
        return fail(MTX_EINVAL, "without x there is no addition: h_out, post_w and gate must be NULL");
    if (!y && (!h_out || b.pre_w))
        return fail(MTX_EINVAL, "y is NULL: h_out must be there and pre_w must not");
    if (y && !b.pre_w) return fail(MTX_EINVAL, "y needs pre_w");
    if (b.rows == 0) return MTX_OK;
    if (!h) return fail(MTX_EINVAL, "h must not be NULL");
    const size_t es = type_size(d->dtype);
    for (const void* p : {h, x, (const void*)h_out, (const void*)y})
        if (!aligned(p, es)) return fail(MTX_EINVAL, "tensors must be aligned to their element size");
    if (!aligned(stats, 16)) return fail(MTX_EINVAL, "stats must be 16-byte aligned");
    if (spans_overlap({rows_span(h == h_out ? nullptr : h, b.rows, b.D, b.ld_h, es, false),
                       rows_span(x, b.rows, b.D, b.ld_x, es, false),
                       rows_span(h_out, b.rows, b.D, b.ld_h, es, true),
                       rows_span(y, b.rows, b.D, b.ld_y, es, true),
                       Span{stats, stats ? (size_t)b.rows * 16 : 0, true}, NORM_PARAM_SPANS(b)}))
        return fail(MTX_EINVAL, "an output overlaps another tensor");
    HIP_TRY(block_norm_fwd(b, h, x, h_out, y, stats, static_cast<hipStream_t>(stream)),
            "mtx_block_norm_forward");
    return MTX_OK;
}

int mtx_block_norm_sizes(const mtx_norm_desc* d, int R, size_t* workspace_bytes)
{
    if (!workspace_bytes) return fail(MTX_EINVAL, "workspace_bytes is NULL");
    BlockNorm b{};
    const int rc = check_norm(d, b);
    if (rc) return rc;
    if (R < 1 || R > 65536 || b.rows % R)
        return fail(MTX_EINVAL, "R must lie in 1 .. 65536 and divide rows");
    if (b.gate_rows && (b.rows / R) % b.gate_rows)
        return fail(MTX_EINVAL, "gate_rows must divide the rows of a shard");
    *workspace_bytes = block_norm_bwd_bytes(b, R);
    return MTX_OK;
}

int mtx_block_norm_backward(const mtx_norm_desc* d, int R, const void* h_out, const void* x,
                            const float* stats, const void* dy, const void* dh_out, void* dh,
                            void* dx, float* d_post_w, float* d_post_b, float* d_gate,
                            float* d_pre_w, float* d_pre_b, size_t ld, void* workspace,
                            size_t workspace_bytes, void* stream)
{
    BlockNorm b{};
    const int rc = check_norm(d, b);
    if (rc) return rc;
    if (R < 1 || R > 65536 || b.rows % R)
        return fail(MTX_EINVAL, "R must lie in 1 .. 65536 and divide rows");
    if (b.gate_rows && (b.rows / R) % b.gate_rows)
        return fail(MTX_EINVAL, "gate_rows must divide the rows of a shard");
    if (dy && !b.pre_w) return fail(MTX_EINVAL, "dy needs pre_w");
    if ((d_post_w && !b.post_w) || (d_post_b && !b.post_b) || (d_gate && !b.gate) ||
        (d_pre_w && !(b.pre_w && dy)) || (d_pre_b && !(b.pre_b && dy)))
        return fail(MTX_EINVAL, "a gradient of an absent operand is asked for");
    const bool want_x = dx || d_post_w || d_post_b || d_gate;
    // (a gradient of the bias, of x without a norm or gate needs only dH)
    if (b.rows) {
        if (!dy && !dh_out) return fail(MTX_EINVAL, "dy and dh_out are both NULL");
        if (want_x && !x) return fail(MTX_EINVAL, "x must not be NULL for its side's gradients");
        if (dy && !h_out) return fail(MTX_EINVAL, "h_out must not be NULL with dy");
        if (!stats && (dy || (want_x && b.post_w))) return fail(MTX_EINVAL, "stats must not be NULL");
    }
    const size_t es = type_size(d->dtype);
    for (const void* p : {h_out, x, dy, dh_out, (const void*)dh, (const void*)dx})
        if (!aligned(p, es)) return fail(MTX_EINVAL, "tensors must be aligned to their element size");
    for (const float* p : {d_post_w, d_post_b, d_gate, d_pre_w, d_pre_b})
        if (!aligned(p, 4)) return fail(MTX_EINVAL, "gradients must be 4-byte aligned");
    if (!aligned(stats, 16)) return fail(MTX_EINVAL, "stats must be 16-byte aligned");
    if (ld < (size_t)b.D) return fail(MTX_EINVAL, "ld must be >= D");
    if (ld > ((size_t)1 << 60) / R) return fail(MTX_EINVAL, "sizes overflow");
    const size_t need = block_norm_bwd_bytes(b, R);
    if (!workspace || !aligned(workspace, 16))
        return fail(MTX_EINVAL, "the workspace must be 16-byte aligned and not NULL");
    if (workspace_bytes < need)
        return fail(MTX_ENOMEM, "workspace too small: %zu bytes given, %zu needed",
                    workspace_bytes, need);
    // the gradients of several parameters may share rows of one vector [R][ld], each at its own columns
    const Span params[] = {rows_span(d_post_w, R, b.D, ld, 4, true), rows_span(d_post_b, R, b.D, ld, 4, true),
                           b.gate_rows ? rows_span(d_gate, b.rows / b.gate_rows, b.D, b.D, 4, true)
                                       : rows_span(d_gate, R, b.D, ld, 4, true),
                           rows_span(d_pre_w, R, b.D, ld, 4, true), rows_span(d_pre_b, R, b.D, ld, 4, true)};
    if (spans_overlap(params)) return fail(MTX_EINVAL, "parameter gradients overlap");
    const Span in_out[] = {rows_span(h_out, b.rows, b.D, b.ld_h, es, false),
                           rows_span(x, b.rows, b.D, b.ld_x, es, false),
                           rows_span(dy, b.rows, b.D, b.ld_y, es, false),
                           rows_span(dh_out == dh ? nullptr : dh_out, b.rows, b.D, b.ld_h, es, false),
                           rows_span(dh, b.rows, b.D, b.ld_h, es, true),
                           rows_span(dx, b.rows, b.D, b.ld_x, es, true),
                           Span{stats, stats ? (size_t)b.rows * 16 : 0, false},
                           Span{workspace, need, true}, NORM_PARAM_SPANS(b)};
    if (spans_overlap(in_out)) return fail(MTX_EINVAL, "an output overlaps another tensor");
    for (const Span& p : params)
        for (const Span& a : in_out)
            if (share_bytes(p, a))
                return fail(MTX_EINVAL, "a parameter gradient overlaps another tensor");
    const BlockNormGrads g{h_out, want_x ? x : nullptr, stats, dy, dh_out, dh, dx, d_post_w, d_post_b, d_gate,
                           d_pre_w, d_pre_b, (long long)ld, false};
    HIP_TRY(block_norm_bwd(b, R, g, workspace, static_cast<hipStream_t>(stream)),
            "mtx_block_norm_backward");
    return MTX_OK;
}

int mtx_average_clip(const float* grads, int R, size_t n, size_t ld, float max_norm, float* avg,
                     float* norm_out, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!grads || !avg) return fail(MTX_EINVAL, "grads and avg must not be NULL");
    if (R < 1) return fail(MTX_EINVAL, "R must be >= 1 (got %d)", R);
    if (n < 1) return fail(MTX_EINVAL, "n must be >= 1");
    if (ld < n) return fail(MTX_EINVAL, "ld must be >= n");
    if (ld > ((size_t)1 << 60) / R) return fail(MTX_EINVAL, "sizes overflow");
    if (!(max_norm > 0.0f)) return fail(MTX_EINVAL, "max_norm must be > 0");
    if (!aligned(grads, 4) || !aligned(avg, 4) || !aligned(norm_out, 4))
        return fail(MTX_EINVAL, "pointers must be 4-byte aligned");
    if (!workspace || !aligned(workspace, 16))
        return fail(MTX_EINVAL, "the workspace must be 16-byte aligned and not NULL");
    if (workspace_bytes < MTX_CLIP_WORKSPACE_BYTES)
        return fail(MTX_ENOMEM, "workspace too small: %zu bytes given, %d needed",
                    workspace_bytes, MTX_CLIP_WORKSPACE_BYTES);
    if (spans_overlap({rows_span(grads, R, n, ld, 4, false), Span{avg, n * 4, true},
                       Span{norm_out, norm_out ? (size_t)4 : 0, true},
                       Span{workspace, MTX_CLIP_WORKSPACE_BYTES, true}}))
        return fail(MTX_EINVAL, "grads, avg, norm_out and the workspace must not overlap");
    HIP_TRY(average_clip(grads, R, n, ld, false, max_norm, avg, norm_out, nullptr,
                         static_cast<double*>(workspace), static_cast<hipStream_t>(stream)),
            "mtx_average_clip");
    return MTX_OK;
}

}  // extern "C"

struct mtx_clip {
    int chunks;
    std::vector<std::pair<uintptr_t, uintptr_t>> spans;   // what the handle uses: disjoint, ascending
    bool in_place;   // every dst is its src or NULL: nothing to write where nothing is clipped
    double* part;
    ClipChunk* table;
    hipStream_t last_stream;   // of the last call that was not captured
};

// Chunks of a list: pieces of at most kClipChunk elements.
static int clip_chunks(const mtx_tensor* t, int count, size_t& chunks)
{
    if (!t || count < 1) return fail(MTX_EINVAL, "the list of tensors is empty");
    chunks = 0;
    for (int i = 0; i < count; ++i) {
        if (!known_type(t[i].src_type) || (t[i].dst && !known_type(t[i].dst_type)))
            return fail(MTX_EINVAL, "tensor %d: types must be MTX_F32 or MTX_BF16", i);
        if (t[i].n > ((size_t)1 << 44)) return fail(MTX_EINVAL, "tensor %d: too large", i);
        if (t[i].n && !t[i].src) return fail(MTX_EINVAL, "tensor %d: src is NULL", i);
        if (t[i].dst == t[i].src && t[i].dst && t[i].dst_type != t[i].src_type)
            return fail(MTX_EINVAL, "tensor %d: clipped in place, its types must be the same", i);
        if (!aligned(t[i].src, type_size(t[i].src_type)) ||
            (t[i].dst && !aligned(t[i].dst, type_size(t[i].dst_type))))
            return fail(MTX_EINVAL, "tensor %d: pointers must be aligned to their element size", i);
        chunks += (t[i].n + kClipChunk - 1) / kClipChunk;
    }
    if (chunks > 2147483647) return fail(MTX_EINVAL, "the list is too large");
    // no written tensor may touch another one: sorted by address, a span that starts before the
    // furthest end so far overlaps an earlier one
    struct Piece {
        uintptr_t beg, end;
        bool written;
    };
    std::vector<Piece> v;
    for (int i = 0; i < count; ++i) {
        if (!t[i].n) continue;
        const uintptr_t s = reinterpret_cast<uintptr_t>(t[i].src),
                        d = reinterpret_cast<uintptr_t>(t[i].dst);
        if (t[i].dst != t[i].src) v.push_back({s, s + t[i].n * type_size(t[i].src_type), false});
        if (t[i].dst) v.push_back({d, d + t[i].n * type_size(t[i].dst_type), true});
    }
    std::sort(v.begin(), v.end(), [](const Piece& a, const Piece& b) { return a.beg < b.beg; });
    uintptr_t end_any = 0, end_written = 0;
    for (const Piece& p : v) {
        if (p.beg < end_written || (p.written && p.beg < end_any))
            return fail(MTX_EINVAL, "a dst overlaps another tensor of the list");
        end_any = std::max(end_any, p.end);
        if (p.written) end_written = std::max(end_written, p.end);
    }
    return MTX_OK;
}

static size_t clip_bytes(size_t chunks)
{
    return align_up(kClipBlocks * sizeof(double), kAlign) +
           align_up(std::max<size_t>(chunks, 1) * sizeof(ClipChunk), kAlign);
}

extern "C" {

int mtx_clip_sizes(const mtx_tensor* tensors, int count, size_t* workspace_bytes)
{
    if (!workspace_bytes) return fail(MTX_EINVAL, "workspace_bytes is NULL");
    try {
        size_t chunks = 0;
        const int rc = clip_chunks(tensors, count, chunks);
        if (rc) return rc;
        *workspace_bytes = clip_bytes(chunks);
        return MTX_OK;
    } catch (...) {
        return fail(MTX_ENOMEM, "host allocation failed");
    }
}

int mtx_init_clip(const mtx_tensor* tensors, int count, void* workspace, size_t workspace_bytes,
                  void* stream, mtx_clip** out)
{
    if (!out) return fail(MTX_EINVAL, "out is NULL");
    *out = nullptr;
    try {
        size_t chunks = 0;
        const int rc = clip_chunks(tensors, count, chunks);
        if (rc) return rc;
        const size_t need = clip_bytes(chunks);
        if (!workspace || !aligned(workspace, kAlign))
            return fail(MTX_EINVAL, "the workspace must be 256-byte aligned and not NULL");
        if (workspace_bytes < need)
            return fail(MTX_ENOMEM, "workspace too small: %zu bytes given, %zu needed",
                        workspace_bytes, need);
        if (being_captured(static_cast<hipStream_t>(stream)))
            return fail(MTX_EINVAL, "the stream is being captured: make the handle before");
        std::vector<ClipChunk> table;
        table.reserve(chunks);
        bool in_place = true;
        for (int i = 0; i < count; ++i) {
            const mtx_tensor& t = tensors[i];
            if (!t.n) continue;
            const size_t es = type_size(t.src_type), ed = t.dst ? type_size(t.dst_type) : 0;
            if (overlap(workspace, need, t.src, t.n * es) ||
                (t.dst && overlap(workspace, need, t.dst, t.n * ed)))
                return fail(MTX_EINVAL, "tensor %d overlaps the workspace", i);
            in_place = in_place && (!t.dst || t.dst == t.src);
            for (size_t o = 0; o < t.n; o += kClipChunk) {
                ClipChunk k{};
                k.src = static_cast<const char*>(t.src) + o * es;
                k.dst = t.dst ? static_cast<char*>(t.dst) + o * ed : nullptr;
                k.n = (unsigned)std::min(kClipChunk, t.n - o);
                k.src_bf16 = t.src_type == MTX_BF16;
                k.dst_bf16 = t.dst && t.dst_type == MTX_BF16;
                const size_t ea = k.dst ? ed : es;
                const size_t off = reinterpret_cast<uintptr_t>(k.dst ? k.dst : k.src) % 16;
                k.head = (unsigned char)std::min<size_t>(k.n, off ? (16 - off) / ea : 0);
                table.push_back(k);
            }
        }
        std::vector<std::pair<uintptr_t, uintptr_t>> spans;
        auto add_span = [&](const void* p, size_t bytes) {
            const uintptr_t a = reinterpret_cast<uintptr_t>(p);
            if (p && bytes) spans.emplace_back(a, a + bytes);
        };
        add_span(workspace, need);
        for (int i = 0; i < count; ++i) {
            add_span(tensors[i].src, tensors[i].n * type_size(tensors[i].src_type));
            if (tensors[i].dst)
                add_span(tensors[i].dst, tensors[i].n * type_size(tensors[i].dst_type));
        }
        std::sort(spans.begin(), spans.end());
        size_t kept = 0;
        for (const auto& p : spans) {
            if (kept && p.first <= spans[kept - 1].second)
                spans[kept - 1].second = std::max(spans[kept - 1].second, p.second);
            else
                spans[kept++] = p;
        }
        spans.resize(kept);
        mtx_clip* c = new mtx_clip;
        c->spans = std::move(spans);
        c->chunks = (int)table.size();
        c->in_place = in_place;
        c->part = static_cast<double*>(workspace);
        c->table = reinterpret_cast<ClipChunk*>(static_cast<char*>(workspace) +
                                                align_up(kClipBlocks * sizeof(double), kAlign));
        c->last_stream = static_cast<hipStream_t>(stream);
        hipError_t e = hipSuccess;
        if (!table.empty())
            e = hipMemcpyAsync(c->table, table.data(), table.size() * sizeof(ClipChunk),
                               hipMemcpyHostToDevice, c->last_stream);
        if (e == hipSuccess) e = hipStreamSynchronize(c->last_stream);
        if (e != hipSuccess) {
            delete c;
            return hip_fail(e, "mtx_init_clip");
        }
        *out = c;
        return MTX_OK;
    } catch (...) {
        return fail(MTX_ENOMEM, "host allocation failed");
    }
}

int mtx_clip_grads(mtx_clip* c, float max_norm, float* norm_out, void* stream)
{
    if (!c) return fail(MTX_EINVAL, "the handle is NULL");
    if (!(max_norm > 0.0f)) return fail(MTX_EINVAL, "max_norm must be > 0");
    if (!aligned(norm_out, 4)) return fail(MTX_EINVAL, "norm_out must be 4-byte aligned");
    if (norm_out) {
        const uintptr_t a = reinterpret_cast<uintptr_t>(norm_out);
        // the last span that begins before norm_out ends
        auto it = std::lower_bound(c->spans.begin(), c->spans.end(), std::make_pair(a + 4, (uintptr_t)0));
        if (it != c->spans.begin() && (--it)->second > a)
            return fail(MTX_EINVAL, "norm_out overlaps a tensor of the list or the workspace");
    }
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (s != c->last_stream && !being_captured(s)) c->last_stream = s;
    HIP_TRY(clip_list(c->table, c->chunks, c->in_place, max_norm, norm_out, c->part, s),
            "mtx_clip_grads");
    return MTX_OK;
}

void mtx_free_clip(mtx_clip* c)
{
    if (!c) return;
    finish_stream(c->last_stream);   // its kernels read the caller's workspace
    delete c;
}

}  // extern "C"
