"""Operands that are columns of one matrix, or lie between another one's rows: accepted, with the
bits of a call on tensors of their own, wherever they share no element; refused where they do."""
import random

import pytest
import torch

from paper_1704_04560_amd import mtx
from tests.ops_ref import BF16, F32

pytestmark = pytest.mark.gpu
MT = {F32: mtx.MTX_F32, BF16: mtx.MTX_BF16}


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _params(g, D):
    return {k: torch.randn(D, generator=g).cuda() for k in ("post_w", "post_b", "gate", "pre_w", "pre_b")}


def _desc(dtype, N, D, p, ld=0):
    return mtx.make_norm_desc(mtx.MTX_NORM_LAYER, MT[dtype], N, D, 1e-5, 0.5, 0, p["post_w"],
                              p["post_b"], p["gate"], p["pre_w"], p["pre_b"], ld, ld, ld)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,D,gap", [(1, 8, 0), (7, 64, 0), (130, 63, 1), (33, 300, 4), (9, 2048, 8)])
def test_block_norm_over_columns(N, D, gap, dtype):
    """The stream, the block's output, the sum and the norm side by side in one matrix; then the
    four gradients in another."""
    print(f"[case] columns N={N} D={D} gap={gap} {dtype}", flush=True)
    g = _gen(N + D)
    p, R = _params(g, D), 1
    ld = 4 * D + gap

    def matrix():
        m = torch.randn(N, ld, generator=g).to(dtype).cuda()
        return m, [m[:, i * D:(i + 1) * D] for i in range(4)]

    A, (h, x, H, y) = matrix()
    G, (dy, dho, dh, dx) = matrix()
    tail = A[:, 4 * D:].clone(), G[:, 4 * D:].clone()
    # a matrix for each operand, at the same place in it: the same path through the kernels
    own = [m.clone()[:, i * D:(i + 1) * D] for m in (A, G) for i in range(4)]
    d = _desc(dtype, N, D, p, ld)
    ws = torch.empty(mtx.mtx_block_norm_sizes(d, R), dtype=torch.uint8, device="cuda")
    res = []
    for t in ((h, x, H, y, dy, dho, dh, dx), own):
        st, gr = torch.empty(N, 4, device="cuda"), torch.empty(5, D, device="cuda")
        mtx.mtx_block_norm_forward(d, t[0], t[1], t[2], t[3], st)
        mtx.mtx_block_norm_backward(d, R, t[2], t[1], st, t[4], t[5], t[6], t[7], *gr, D, ws)
        torch.cuda.synchronize()
        res.append([q.clone() for q in t] + [st, gr])
    for a, b in zip(*res):
        assert torch.equal(a, b)
    assert torch.equal(A[:, 4 * D:], tail[0]) and torch.equal(G[:, 4 * D:], tail[1])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,D,group", [(9, 8, 3), (130, 64, 0), (64, 120, 4), (1100, 256, 1), (33, 1000, 0),
                                       (12, 4096, 2)])
def test_strides_of_their_own(N, D, group, dtype):
    """The stream, the block's output and the norm with three strides: the bits of packed rows."""
    print(f"[case] strides N={N} D={D} group={group} {dtype}", flush=True)
    g = _gen(N * D)
    p = _params(g, D)
    p["gate"] = torch.randn(N // group if group else 1, D, generator=g).cuda()
    t = [torch.randn(N, D, generator=g).to(dtype).cuda() for _ in range(4)]   # h, x, dy, dh_out
    res = []
    for lh, lx, ly in ((D + 8, 2 * D + 40, D + 24), (D, D, D)):
        def rows(ld, src=None):
            m = torch.full((N, ld), 3.0, dtype=dtype, device="cuda")
            if src is not None:
                m[:, :D] = src
            return m

        d = mtx.make_norm_desc(mtx.MTX_NORM_LAYER, MT[dtype], N, D, 1e-5, 0.5, group, p["post_w"],
                               p["post_b"], p["gate"], p["pre_w"], p["pre_b"], lh, lx, ly)
        h, x, H, y = rows(lh, t[0]), rows(lx, t[1]), rows(lh), rows(ly)
        dy, dho, dh, dx = rows(ly, t[2]), rows(lh, t[3]), rows(lh), rows(lx)
        st, gr, gg = (torch.empty(N, 4, device="cuda"), torch.empty(5, D, device="cuda"),
                      torch.empty_like(p["gate"]))
        ws = torch.empty(mtx.mtx_block_norm_sizes(d, 1), dtype=torch.uint8, device="cuda")
        mtx.mtx_block_norm_forward(d, h, x, H, y, st)
        mtx.mtx_block_norm_backward(d, 1, H, x, st, dy, dho, dh, dx, gr[0], gr[1], gg, gr[3], gr[4], D, ws)
        torch.cuda.synchronize()
        assert all((m[:, D:] == 3.0).all() for m in (h, x, H, y, dy, dho, dh, dx))
        res.append([m[:, :D].clone() for m in (H, y, dh, dx)] + [st, gr[[0, 1, 3, 4]], gg])
    for a, b in zip(*res):
        assert torch.equal(a, b)


def test_every_placement_of_rows():
    """Random places and strides in one small buffer, against a comparison of every element."""
    rng = random.Random(5)
    N, D, size = 5, 5, 400
    g = _gen(1)
    p = {k: None for k in ("post_w", "post_b", "gate")} | {"pre_w": torch.randn(D, generator=g).cuda(),
                                                           "pre_b": None}
    taken = refused = 0
    for _ in range(400):
        ld = [rng.choice([D, 2 * D, 3 * D, 17, 20, rng.randint(D, 40)]) for _ in range(2)]
        h, x, H, y = (rng.randint(0, size - N * 40) for _ in range(4))
        if rng.random() < 0.5:   # columns of one matrix
            ld = [20, 20]
            h, x, H, y = (h + c * D for c in rng.sample(range(4), 4))
        cells = [set((o + i * l + j) for i in range(N) for j in range(D))
                 for o, l in ((h, ld[0]), (x, ld[0]), (H, ld[0]), (y, ld[1]))]
        clash = any(cells[a] & cells[b] for a, b in ((0, 2), (0, 3), (1, 2), (1, 3), (2, 3)))
        buf = torch.randn(size, generator=g).cuda()
        was = buf.clone()
        d = mtx.make_norm_desc(mtx.MTX_NORM_RMS, mtx.MTX_F32, N, D, 1e-5, 1.0, 0, None, None, None,
                               p["pre_w"], None, ld[0], ld[0], ld[1])

        def call(b):
            mtx.mtx_block_norm_forward(d, b[h:], b[x:], b[H:], b[y:], None)

        if h == H and not any(cells[a] & cells[b] for a, b in ((1, 2), (0, 3), (1, 3), (2, 3))):
            clash = False   # the stream in place
        if clash:
            refused += 1
            with pytest.raises(mtx.MtxError) as e:
                call(buf)
            assert e.value.code == mtx.MTX_EINVAL
            assert torch.equal(buf, was)
            continue
        taken += 1
        call(buf)

        def rows(b, o, l):
            return torch.as_strided(b, (N, D), (l, 1), o)

        Ho, yo = torch.empty(N, D, device="cuda"), torch.empty(N, D, device="cuda")
        own = mtx.make_norm_desc(mtx.MTX_NORM_RMS, mtx.MTX_F32, N, D, 1e-5, 1.0, 0, None, None, None,
                                 p["pre_w"], None)
        mtx.mtx_block_norm_forward(own, rows(was, h, ld[0]).contiguous(),
                                   rows(was, x, ld[0]).contiguous(), Ho, yo, None)
        rows(was, H, ld[0]).copy_(Ho)
        rows(was, y, ld[1]).copy_(yo)
        assert torch.equal(buf, was)
    assert taken > 50 and refused > 50


def test_average_and_norm_between_the_rows():
    """The average in columns of the gradient rows' own matrix, the norm in their padding."""
    R, n = 3, 1001
    buf = torch.randn(R, 2 * n + 7, generator=_gen(3)).cuda()
    own = buf[:, :n].contiguous()
    avg, nrm = torch.empty(n, device="cuda"), torch.empty(1, device="cuda")
    ws = torch.empty(mtx.MTX_CLIP_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    mtx.mtx_average_clip(own, R, n, n, 0.5, avg, nrm, ws)
    mtx.mtx_average_clip(buf, R, n, 2 * n + 7, 0.5, buf[1, n:], buf[2, 2 * n:], ws)
    torch.cuda.synchronize()
    assert torch.equal(buf[1, n:2 * n], avg) and torch.equal(buf[2, 2 * n], nrm[0])
    assert torch.equal(buf[:, :n], own)
    with pytest.raises(mtx.MtxError):
        mtx.mtx_average_clip(buf, R, n, 2 * n + 7, 0.5, buf[1, n + 8:], None, ws)


def test_embedding_beside_other_columns():
    """Rows of y beside the rows of dy; a shard's gradient beside the next shard's padding."""
    V, D, n, R = 50, 24, 60, 2
    g = _gen(4)
    w = torch.randn(V, D, generator=g).cuda()
    tok = torch.randint(0, V, (n,), generator=g, dtype=torch.int32).cuda()
    m = torch.randn(n, 2 * D, generator=g).cuda()
    dy = m[:, :D].contiguous()
    mtx.mtx_embed_forward(w, mtx.MTX_F32, V, D, tok, n, -1, 2.0, m[:, D:], mtx.MTX_F32, 2 * D)
    assert torch.equal(m[:, D:], 2 * w[tok.long()]) and torch.equal(m[:, :D], dy)
    # grads and dy in the rows of one matrix
    ld = V * D + n // R * D
    both = torch.zeros(R, ld, device="cuda")
    t2 = tok[:R].contiguous()
    both[0, V * D:V * D + R * D] = dy[:R].reshape(-1)
    ws = torch.empty(mtx.mtx_embed_sizes(1, R, V, D), dtype=torch.uint8, device="cuda")
    mtx.mtx_embed_backward(t2, 1, R, both[0, V * D:], mtx.MTX_F32, D, V, D, -1, 1.0, both, ld, False, ws)
    torch.cuda.synchronize()
    for r in range(R):
        want = torch.zeros(V, D, device="cuda")
        want[t2[r].long()] = dy[r]
        assert torch.equal(both[r, :V * D].view(V, D), want)
