"""Block norms on the GPU (post-norm, gate, residual addition, pre-norm in one pass, and their
gradients) against 64-bit forms and differences, through the C ABI."""
import pytest
import torch

from paper_1704_04560_amd import mtx
from tests.ops_ref import BF16, F32, U, Norm, assert_within, half

pytestmark = pytest.mark.gpu
MT = {F32: mtx.MTX_F32, BF16: mtx.MTX_BF16}
EPS = 1e-5


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _params(g, D, layer, post, gate, G):
    def w(mean, *s):
        return mean + 0.3 * torch.randn(*s, generator=g)
    p = {"pre_w": w(1.0, D), "pre_b": w(0.0, D) if layer else None,
         "post_w": w(1.0, D) if post else None, "post_b": w(0.0, D) if post and layer else None,
         "gate": w(0.2, G, D) if gate else None}
    return p


def _strided(t, ld, off):
    N, D = t.shape
    buf = torch.full((N * ld + off + 16,), 5.0, dtype=t.dtype, device="cuda")
    v = buf[off:off + N * ld].view(N, ld)
    v[:, :D] = t.cuda()
    return v


def _dev(p):
    return {k: None if v is None else v.cuda() for k, v in p.items()}


def _dbl(p):
    return {k: None if v is None else v.double() for k, v in p.items()}


def _desc(kind, dtype, N, D, scale, group, p, ld=(0, 0, 0)):
    return mtx.make_norm_desc(kind, MT[dtype], N, D, EPS, scale, group, p["post_w"], p["post_b"],
                              p["gate"], p["pre_w"], p["pre_b"], *ld)


DIMS = [  # rows, D, shards, rows of a gate (0: one gate), extra strides, offset
    (1, 1, 1, 0, 0, 0), (3, 2, 3, 1, 0, 0), (5, 63, 1, 0, 3, 1), (8, 64, 2, 2, 0, 0),
    (6, 65, 2, 3, 0, 0), (70, 300, 2, 7, 4, 0), (33, 771, 3, 11, 5, 1), (260, 128, 4, 65, 8, 0),
    (12, 1024, 1, 0, 0, 0), (130, 2056, 2, 5, 0, 0), (9, 4096, 3, 0, 8, 0), (5, 5001, 1, 0, 0, 0),
    (4, 8192, 2, 1, 0, 0), (3, 16384, 1, 0, 0, 0), (2, 16383, 1, 2, 1, 1), (1100, 40, 2, 0, 0, 0),
    (4097, 16, 1, 0, 0, 0), (520, 513, 1, 520, 0, 0), (1200, 64, 3, 2, 0, 0), (999, 100, 3, 3, 4, 1),
    (2048, 128, 2, 16, 0, 0), (4100, 24, 4, 1, 0, 0), (300, 200, 2, 5, 8, 0), (5001, 96, 1, 0, 0, 0),
    (2310, 252, 2, 33, 4, 0), (7000, 8, 2, 7, 0, 0)]
FORMS = [  # layer norm, post norm, gate, x
    (False, True, True, True), (True, True, True, True), (False, True, False, True),
    (True, False, True, True), (False, False, False, True), (True, False, False, False),
    (False, False, False, False)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("layer,post,gate,has_x", FORMS)
@pytest.mark.parametrize("N,D,R,group,extra,off", DIMS)
def test_forward_and_backward(N, D, R, group, extra, off, layer, post, gate, has_x, dtype):
    group = group if gate else 0
    print(f"[case] block_norm N={N} D={D} R={R} group={group} layer={layer} post={post} "
          f"gate={gate} x={has_x} {dtype} ld={D + extra}", flush=True)
    g = _gen(N * 7 + D)
    p = _params(g, D, layer, post, gate, N // group if group else 1)
    kind = mtx.MTX_NORM_LAYER if layer else mtx.MTX_NORM_RMS
    scale, ld = 0.75, D + extra
    ref = Norm(layer, EPS, scale, group, _dbl(p), R)

    def draw(mean=0.0, std=1.0):
        return (mean + std * torch.randn(N, D, generator=g)).to(dtype)

    h, x = draw(0.5), draw(-0.3) if has_x else None
    if N > 2:   # a row of zeros, and one far from zero
        h[1] = 0.0
        h[2] += 20.0
        if has_x:
            x[1] = 0.0
    pd = _dev(p)
    d = _desc(kind, dtype, N, D, scale, group, pd, (ld, ld, ld))
    hd, xd = _strided(h, ld, off), None if x is None else _strided(x, ld, off)
    h_out = _strided(torch.zeros(N, D, dtype=dtype), ld, off) if has_x else None
    y = _strided(torch.zeros(N, D, dtype=dtype), ld, off)
    st = torch.full((N, 4), 9.0, device="cuda")
    mtx.mtx_block_norm_forward(d, hd, xd, h_out, y, st)
    torch.cuda.synchronize()
    v, m = ref.forward(h.double(), None if x is None else x.double())
    k = U * (D / 64 + 32)
    if has_x:
        assert_within(h_out[:, :D], v["h"], k * m["h"] + half(dtype) * v["h"].abs(), "h_out")
    assert_within(y[:, :D], v["y"], 2 * k * m["y"] + half(dtype) * v["y"].abs(), "y")
    cols = [0, 1, 2, 3] if post else [2, 3]
    assert_within(st[:, cols], v["st"][:, cols], 2 * k * m["st"][:, cols], "stats")
    for t in (h_out, y):
        assert t is None or (t[:, D:] == 5.0).all(), "gaps between rows"
    if not post:
        assert (st[:, :2] == 9.0).all()

    # backward, from the reference's statistics and the rounded stream
    H = v["h"].to(dtype)
    stats = v["st"].float()
    dy, dho = draw(0.1, 0.5), draw(0.0, 0.7)
    want, mag = ref.backward(H.double(), None if x is None else x.double(), stats.double(),
                             dy.double(), dho.double())
    names = ["pre_w"] + (["pre_b"] if layer else [])
    if has_x:
        names += (["post_w"] if post else []) + (["post_b"] if post and layer else [])
        names += ["gate"] if gate else []
    row = len(names) * D + 3
    grads = torch.full((R, row), 3.0, device="cuda")
    slot = {n: grads[:, i * D:(i + 1) * D] for i, n in enumerate(names)}
    dgate = torch.full((N // group, D), 3.0, device="cuda") if group and has_x else slot.get("gate")
    dh, dx = (_strided(torch.zeros(N, D, dtype=dtype), ld, off) for _ in range(2))
    ws = torch.empty(mtx.mtx_block_norm_sizes(d, R), dtype=torch.uint8, device="cuda")

    def back(dh_, dx_, out):
        mtx.mtx_block_norm_backward(
            d, R, _strided(H, ld, off), xd, stats.cuda(), _strided(dy, ld, off),
            out, dh_, dx_, slot.get("post_w"), slot.get("post_b"), dgate if gate and has_x else None,
            slot["pre_w"], slot.get("pre_b"), row, ws)

    dod = _strided(dho, ld, off)
    back(dh, dx if has_x else None, dod)
    torch.cuda.synchronize()
    assert_within(dh[:, :D], want["dh"], k * mag["dh"] + half(dtype) * want["dh"].abs(), "dh")
    if has_x:
        assert_within(dx[:, :D], want["dx"], 2 * k * mag["dx"] + half(dtype) * want["dx"].abs(), "dx")
    kr = U * (N // R + D / 64 + 32)
    for n in names:
        got = dgate if n == "gate" and group else slot[n]
        assert_within(got, want[n], 2 * kr * mag[n], n)
    assert (grads[:, len(names) * D:] == 3.0).all() and (dh[:, D:] == 5.0).all()
    # the same bits again, with dh written over dh_out and no dx
    first = [dh.clone(), grads.clone()] + ([dgate.clone()] if gate and has_x else [])
    back(dod, None, dod)
    again = [dod, grads] + ([dgate] if gate and has_x else [])
    assert all(torch.equal(a[..., :D], b[..., :D]) for a, b in zip(first, again))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,D", [(7, 96), (3, 2048), (600, 770)])
def test_partial_calls(N, D, dtype):
    """In place, without the next norm, without a gradient of one side: the same bits as the whole
    call, where it computes the same."""
    g = _gen(N + D)
    p = _dev(_params(g, D, False, True, True, 1))
    h, x = (torch.randn(N, D, generator=g).to(dtype).cuda() for _ in range(2))
    d = _desc(mtx.MTX_NORM_RMS, dtype, N, D, 1.0, 0, p)
    H, y, st = torch.empty_like(h), torch.empty_like(h), torch.empty(N, 4, device="cuda")
    mtx.mtx_block_norm_forward(d, h, x, H, y, st)
    inplace, y2 = h.clone(), torch.empty_like(h)
    mtx.mtx_block_norm_forward(d, inplace, x, inplace, y2, None)
    assert torch.equal(inplace, H) and torch.equal(y2, y)
    y3 = torch.empty_like(h)
    mtx.mtx_block_norm_forward(d, h, x, None, y3, None)
    assert torch.equal(y3, y)
    q = dict(p, pre_w=None)
    H4 = torch.empty_like(h)
    mtx.mtx_block_norm_forward(_desc(mtx.MTX_NORM_RMS, dtype, N, D, 1.0, 0, q), h, x, H4, None, None)
    assert torch.equal(H4, H)
    # gradients: dy alone, dh_out alone
    dy, dho = (torch.randn(N, D, generator=g).to(dtype).cuda() for _ in range(2))
    ws = torch.empty(mtx.mtx_block_norm_sizes(d, 1), dtype=torch.uint8, device="cuda")
    zero = torch.zeros_like(dy)
    out = []
    for a, b in ((dy, None), (dy, zero), (None, dho), (zero, dho)):
        dh, dx, gr = torch.empty_like(h), torch.empty_like(h), torch.zeros(3, D, device="cuda")
        mtx.mtx_block_norm_backward(d, 1, H, x, st, a, b, dh, dx, gr[0], None, gr[1],
                                    gr[2] if a is not None else None, None, D, ws)
        out.append((dh, dx, gr))
    for a, b in zip(out[0] + out[2], out[1] + out[3]):
        assert torch.equal(a, b)


def test_gradients_agree_with_differences():
    """Each gradient against central differences of the forward pass (fp32, step 2^-7).  Bound: the
    difference of two fp32 forwards of loss terms L = sum |y w| + |H w| has rounding error below
    64 U L / step; the third-order term is step^2 / 6 times a third derivative, which for rows
    scaled to unit size is below 50 of the gradient's own scale."""
    N, D, step = 4, 24, 2.0 ** -7
    g = _gen(3)
    p = _params(g, D, True, True, True, 1)
    h, x, a, b = (torch.randn(N, D, generator=g) for _ in range(4))   # a, b: the loss's weights
    leaves = {"h": h, "x": x, "post_w": p["post_w"], "post_b": p["post_b"], "gate": p["gate"],
              "pre_w": p["pre_w"], "pre_b": p["pre_b"]}

    def forward(t):
        q = _dev({k: t[k] for k in p})
        d = _desc(mtx.MTX_NORM_LAYER, F32, N, D, 0.5, 0, q)
        H, y, st = (torch.empty(N, D, device="cuda"), torch.empty(N, D, device="cuda"),
                    torch.empty(N, 4, device="cuda"))
        mtx.mtx_block_norm_forward(d, t["h"].cuda(), t["x"].cuda(), H, y, st)
        return d, H, y, st

    def loss(t):
        _, H, y, _ = forward(t)
        return float((y.cpu().double() * a.double()).sum() + (H.cpu().double() * b.double()).sum())

    d, H, y, st = forward(leaves)
    ws = torch.empty(mtx.mtx_block_norm_sizes(d, 1), dtype=torch.uint8, device="cuda")
    got = {k: torch.empty_like(v, device="cuda") for k, v in leaves.items()}
    mtx.mtx_block_norm_backward(d, 1, H, x.cuda(), st, a.cuda(), b.cuda(), got["h"], got["x"],
                                got["post_w"], got["post_b"], got["gate"], got["pre_w"],
                                got["pre_b"], D, ws)
    L = float((y.cpu().abs() * a.abs()).sum() + (H.cpu().abs() * b.abs()).sum())
    for k, v in leaves.items():
        scale = float(got[k].abs().max())
        for i in range(0, v.numel(), 5):
            hi, lo = v.clone(), v.clone()
            hi.view(-1)[i] += step
            lo.view(-1)[i] -= step
            fd = (loss(dict(leaves, **{k: hi})) - loss(dict(leaves, **{k: lo}))) / (2 * step)
            tol = 64 * U * L / step + 50 * step * step / 6 * max(scale, 1.0)
            assert abs(fd - float(got[k].view(-1)[i])) <= tol, (k, i)


def test_bad_rows_stay_alone():
    """A row with an infinity or NaN spoils itself and the parameters' sums, no other row."""
    N, D = 9, 640
    g = _gen(8)
    p = _dev(_params(g, D, False, True, False, 1))
    h, x = (torch.randn(N, D, generator=g).cuda() for _ in range(2))
    d = _desc(mtx.MTX_NORM_RMS, F32, N, D, 1.0, 0, p)
    outs = []
    for bad in (False, True):
        if bad:
            x[4, 7], h[6, 0] = float("inf"), float("nan")
        H, y = torch.empty_like(h), torch.empty_like(h)
        mtx.mtx_block_norm_forward(d, h, x, H, y, None)
        outs.append((H, y))
    keep = [i for i in range(N) if i not in (4, 6)]
    for a, b in zip(*outs):
        assert torch.equal(a[keep], b[keep])
    assert torch.isnan(outs[1][1][4]).any() and torch.isnan(outs[1][1][6]).all()


def test_no_rows():
    p = _dev(_params(_gen(1), 64, True, False, False, 1))
    d = _desc(mtx.MTX_NORM_LAYER, F32, 0, 64, 1.0, 0, p)
    e = torch.empty(1, 64, device="cuda")
    mtx.mtx_block_norm_forward(d, None, None, None, e, None)
    gr = torch.ones(2, 3, 64, device="cuda")
    ws = torch.empty(mtx.mtx_block_norm_sizes(d, 2), dtype=torch.uint8, device="cuda")
    mtx.mtx_block_norm_backward(d, 2, None, None, None, e, None, None, None, None, None, None,
                                gr[0, 0], gr[0, 1], 192, ws)
    torch.cuda.synchronize()
    assert (gr[:, :2] == 0).all() and (gr[:, 2] == 1).all()


def test_captured_and_replayed():
    N, D, R = 515, 384, 5
    g = _gen(2)
    p = _dev(_params(g, D, False, True, True, 1))
    d = _desc(mtx.MTX_NORM_RMS, BF16, N, D, 1.0, 0, p)
    t = [torch.randn(N, D, generator=g).to(BF16).cuda() for _ in range(4)]
    out = [torch.empty_like(t[0]) for _ in range(4)]
    st, gr = torch.empty(N, 4, device="cuda"), torch.empty(R, 3 * D, device="cuda")
    ws = torch.empty(mtx.mtx_block_norm_sizes(d, R), dtype=torch.uint8, device="cuda")

    def step(stream=None):
        mtx.mtx_block_norm_forward(d, t[0], t[1], out[0], out[1], st, stream=stream)
        mtx.mtx_block_norm_backward(d, R, out[0], t[1], st, t[2], t[3], out[2], out[3], gr, None,
                                    gr[:, D:], gr[:, 2 * D:], None, 3 * D, ws, stream=stream)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for q in t:
            q.copy_(torch.randn(N, D, generator=g).to(BF16))
        step()
        torch.cuda.synchronize()
        want = [q.clone() for q in out + [st, gr]]
        for q in out + [st, gr]:
            q.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out + [st, gr]))


def test_many_rows_and_rows_past_32_bits():
    """More rows than one launch takes threads (2^26 + 5 rows of one element), and rows 2^28 apart."""
    N = (1 << 26) + 5
    print(f"[case] block_norm N={N} D=1", flush=True)
    p = _dev(_params(_gen(1), 1, False, False, False, 1))
    d = _desc(mtx.MTX_NORM_RMS, BF16, N, 1, 1.0, 0, p)
    h = torch.arange(N, device="cuda", dtype=torch.float32).remainder_(1000).add_(1).to(BF16).view(N, 1)
    y = torch.zeros_like(h)
    mtx.mtx_block_norm_forward(d, h, None, None, y, None)
    f = h[:1000].double()
    want = f / (f * f + EPS).sqrt() * p["pre_w"].double()
    got = y[:N - N % 1000].view(-1, 1000).float()
    assert (got.amax(0) == got.amin(0)).all()   # every repetition gives the same bits
    assert_within(got[0], want[:, 0], want[:, 0].abs() * (half(BF16) + 8 * U), "y")
    assert torch.equal(y[-(N % 1000):], y[:N % 1000])
    del h, y
    ld, N, D = 1 << 28, 10, 520
    g = _gen(2)
    p = _dev(_params(g, D, True, True, True, 1))
    t = torch.zeros(2, N, ld, dtype=BF16, device="cuda")
    t[:, :, :D] = torch.randn(2, N, D, generator=g).to(BF16).cuda()
    small = t[:, :, :D].contiguous()
    outs = []
    for k, (a, l) in enumerate(((t, ld), (small, D))):
        d = _desc(mtx.MTX_NORM_LAYER, BF16, N, D, 1.0, 0, p, (l, l, l))
        st = torch.empty(N, 4, device="cuda")
        y = torch.zeros_like(a[0])
        mtx.mtx_block_norm_forward(d, a[0], a[1], a[0], y, st)
        gr, ws = torch.empty(5, D, device="cuda"), torch.empty(mtx.mtx_block_norm_sizes(d, 1),
                                                               dtype=torch.uint8, device="cuda")
        dx = torch.zeros_like(a[0])
        mtx.mtx_block_norm_backward(d, 1, a[0], a[1], st, y, None, None, dx, gr[0], gr[1], gr[2],
                                    gr[3], gr[4], D, ws)
        outs.append((a[0][:, :D].clone(), y[:, :D].clone(), dx[:, :D].clone(), st, gr))
    for a, b in zip(*outs):
        assert torch.equal(a, b)
