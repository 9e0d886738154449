"""The operators on caller tensors refuse invalid calls on the host, before anything is enqueued
(these calls need no device; the addresses are never read)."""
import ctypes as C
import math

import numpy as np
import pytest

from paper_1704_04560_amd import mtx

F, B = mtx.MTX_F32, mtx.MTX_BF16
BASE = 1 << 33   # made-up addresses, far apart
A = [BASE + i * (1 << 36) for i in range(16)]


class Buf(int):
    """An address with a size, standing for a workspace tensor."""
    nbytes = 1 << 34


def code(fn, *args):
    with pytest.raises(mtx.MtxError) as e:
        fn(*args, stream=0)
    return e.value.code


def test_embed_forward():
    def call(w=A[0], wt=F, V=10, D=8, tok=A[1], n=4, pad=-1, scale=1.0, y=A[2], yt=B, ldy=8):
        return code(mtx.mtx_embed_forward, w, wt, V, D, tok, n, pad, scale, y, yt, ldy)

    for bad in (dict(w=None), dict(tok=None), dict(y=None), dict(V=0), dict(D=0), dict(wt=2),
                dict(yt=-1), dict(ldy=7), dict(scale=math.nan), dict(n=1 << 31),
                dict(w=A[0] + 2), dict(tok=A[1] + 2), dict(y=A[2] + 1), dict(y=A[0] + 16),
                dict(y=A[1] - 8), dict(ldy=1 << 62),
                dict(D=(1 << 24) + 1, ldy=1 << 25)):
        assert call(**bad) == mtx.MTX_EINVAL, bad


def test_embed_backward():
    size = mtx.mtx_embed_sizes(4, 2, 10, 8)
    assert size > 0

    def call(tok=A[1], n=4, R=2, dy=A[0], dt=B, lddy=8, V=10, D=8, pad=-1, scale=1.0, g=A[2],
             ld=80, acc=False, ws=Buf(A[3])):
        return code(mtx.mtx_embed_backward, tok, n, R, dy, dt, lddy, V, D, pad, scale, g, ld, acc, ws)

    for bad in (dict(tok=None), dict(dy=None), dict(g=None), dict(ws=None), dict(R=0), dict(V=0),
                dict(D=-1), dict(dt=5), dict(lddy=7), dict(ld=79), dict(scale=math.inf),
                dict(n=1 << 30), dict(tok=A[1] + 1), dict(dy=A[0] + 1), dict(g=A[2] + 2),
                dict(ws=Buf(A[3] + 8)), dict(g=A[0] + 64), dict(g=A[3]), dict(dy=A[3] + 16),
                dict(tok=A[2] + 4 * 159), dict(ld=1 << 61), dict(lddy=1 << 61)):
        assert call(**bad) == mtx.MTX_EINVAL, bad
    small = Buf(A[3])
    small.nbytes = size - 1
    assert call(ws=small) == mtx.MTX_ENOMEM
    with pytest.raises(mtx.MtxError):
        mtx.mtx_embed_sizes(1 << 31, 1, 10, 8)


def desc(kind=mtx.MTX_NORM_LAYER, dtype=F, rows=12, D=8, eps=1e-5, scale=1.0, group=0, post_w=A[8],
         post_b=A[9], gate=A[10], pre_w=A[11], pre_b=A[12], ld=(0, 0, 0)):
    return mtx.make_norm_desc(kind, dtype, rows, D, eps, scale, group, post_w, post_b, gate, pre_w,
                              pre_b, *ld)


BAD_DESC = (dict(kind=2), dict(dtype=3), dict(D=0), dict(rows=1 << 31), dict(eps=-1.0),
            dict(eps=math.nan), dict(scale=math.inf), dict(kind=mtx.MTX_NORM_RMS),
            dict(post_w=None), dict(pre_w=None), dict(gate=None, group=3), dict(group=5),
            dict(post_w=A[8] + 1), dict(gate=A[10] + 2), dict(ld=(7, 0, 0)), dict(ld=(0, 4, 0)),
            dict(ld=(0, 0, 1 << 40)))


def test_block_norm_forward():
    def call(h=A[0], x=A[1], h_out=A[2], y=A[3], st=A[4], **kw):
        return code(mtx.mtx_block_norm_forward, desc(**kw), h, x, h_out, y, st)

    for bad in BAD_DESC + (dict(h=None), dict(x=None), dict(y=None), dict(h=A[0] + 2),
                           dict(y=A[3] + 1), dict(st=A[4] + 4), dict(y=A[0]), dict(y=A[1] + 4),
                           dict(h_out=A[1]), dict(h_out=A[0] + 32), dict(y=A[2] + 16),
                           dict(st=A[3] + 16), dict(y=A[11]), dict(h_out=A[8] - 16)):
        assert call(**bad) == mtx.MTX_EINVAL, bad
    assert call(D=16385) == mtx.MTX_EUNSUPPORTED
    none = dict(x=None, h_out=None, post_w=None, post_b=None, gate=None)
    assert call(**none, h=None) == mtx.MTX_EINVAL
    assert call(pre_w=None, pre_b=None) == mtx.MTX_EINVAL          # y without its weight
    assert call(y=None, h_out=None, pre_w=None, pre_b=None) == mtx.MTX_EINVAL
    with pytest.raises(mtx.MtxError):
        mtx._check(mtx.lib().mtx_block_norm_forward(None, None, None, None, None, None, None))


def test_block_norm_backward():
    d = dict(pw=A[13], pb=A[13] + 32, gt=A[13] + 64, qw=A[13] + 96, qb=A[13] + 128, ld=40)
    size = mtx.mtx_block_norm_sizes(desc(), 3)

    def call(R=3, h_out=A[0], x=A[1], st=A[2], dy=A[3], dho=A[4], dh=A[5], dx=A[6], ws=Buf(A[7]),
             pw=d["pw"], pb=d["pb"], gt=d["gt"], qw=d["qw"], qb=d["qb"], ld_=40, **kw):
        return code(mtx.mtx_block_norm_backward, desc(**kw), R, h_out, x, st, dy, dho, dh, dx, pw,
                    pb, gt, qw, qb, ld_, ws)

    for bad in BAD_DESC + (
            dict(R=0), dict(R=5), dict(group=12), dict(x=None), dict(h_out=None), dict(st=None),
            dict(dy=None), dict(dy=None, dho=None, qw=None, qb=None), dict(ws=None),
            dict(ws=Buf(A[7] + 4)), dict(ld_=7), dict(ld_=1 << 61), dict(dh=A[5] + 1),
            dict(st=A[2] + 8), dict(pw=A[13] + 2), dict(dh=A[0]), dict(dx=A[1]), dict(dx=A[5] + 8),
            dict(dh=A[4] + 32), dict(dx=A[4]), dict(pw=A[6] + 64), dict(qb=A[7]), dict(pb=d["pw"]),
            dict(gt=d["pw"] + 28), dict(qw=d["pw"] + 40 * 4 - 4), dict(qb=d["pw"] + 80 * 4 + 28),
            dict(gt=d["qb"] + 4, group=2), dict(gt=A[5], group=2), dict(pw=A[8]),
            dict(post_w=None, post_b=None), dict(gate=None)):
        assert call(**bad) == mtx.MTX_EINVAL, bad
    small = Buf(A[7])
    small.nbytes = size - 1
    assert call(ws=small) == mtx.MTX_ENOMEM
    for R in (0, 5, 65537):
        with pytest.raises(mtx.MtxError):
            mtx.mtx_block_norm_sizes(desc(), R)


def test_average_clip():
    def call(g=A[0], R=3, n=10, ld=12, m=1.0, avg=A[1], nrm=A[2], ws=Buf(A[3])):
        return code(mtx.mtx_average_clip, g, R, n, ld, m, avg, nrm, ws)

    for bad in (dict(g=None), dict(avg=None), dict(ws=None), dict(R=0), dict(n=0), dict(ld=9),
                dict(m=0.0), dict(m=-1.0), dict(m=math.nan), dict(g=A[0] + 1), dict(avg=A[1] + 2),
                dict(nrm=A[2] + 2), dict(ws=Buf(A[3] + 8)), dict(avg=A[0] + 4 * 33),
                dict(nrm=A[1] + 36), dict(nrm=A[3] + 4), dict(ld=1 << 61)):
        assert call(**bad) == mtx.MTX_EINVAL, bad
    small = Buf(A[3])
    small.nbytes = mtx.MTX_CLIP_WORKSPACE_BYTES - 1
    assert call(ws=small) == mtx.MTX_ENOMEM


def tensors(*rows):
    arr = (mtx.mtx_tensor * max(1, len(rows)))()
    for a, r in zip(arr, rows):
        a.src, a.dst, a.n, a.src_type, a.dst_type = r
    return arr


def test_clip_list():
    ok = (A[0], A[1], 100, F, F)
    need = mtx.mtx_clip_sizes(tensors(ok))
    lists = [
        [(None, A[1], 4, F, F)], [(A[0], A[1], 4, 2, F)], [(A[0], A[1], 4, F, 7)],
        [(A[0] + 2, A[1], 4, F, F)], [(A[0], A[1] + 1, 4, F, B)], [(A[0], A[0], 4, F, B)],
        [(A[0], A[0] + 4, 4, F, F)], [ok, ok], [ok, (A[2], A[1] + 396, 1, F, F)],
        [ok, (A[0] + 40, A[0] + 40, 2, F, F)],     # clipped in place inside another's source
        [(A[0], A[0], 8, F, F), (A[0] + 28, None, 1, F, F)],   # read where another is written
        [(A[0], None, 8, F, F), (A[0], A[0], 8, F, F)],
        [(A[0], A[1], 1 << 45, F, F)],
    ]
    for rows in lists:
        with pytest.raises(mtx.MtxError) as e:
            mtx.mtx_clip_sizes(tensors(*rows))
        assert e.value.code == mtx.MTX_EINVAL, rows
        assert code(mtx.mtx_init_clip, tensors(*rows), Buf(A[5])) == mtx.MTX_EINVAL
    # two read-only tensors may share elements; empty tensors may be anywhere
    mtx.mtx_clip_sizes(tensors((A[0], None, 8, F, F), (A[0], None, 8, F, F), (None, None, 0, F, F)))
    out = C.c_size_t()
    assert mtx.lib().mtx_clip_sizes(tensors(ok), 0, C.byref(out)) == mtx.MTX_EINVAL
    assert mtx.lib().mtx_clip_sizes(None, 1, C.byref(out)) == mtx.MTX_EINVAL
    for ws in (None, Buf(A[5] + 16), Buf(A[0] - 256), Buf(A[1])):
        assert code(mtx.mtx_init_clip, tensors(ok), ws) == mtx.MTX_EINVAL
    small = Buf(A[5])
    small.nbytes = need - 1
    assert code(mtx.mtx_init_clip, tensors(ok), small) == mtx.MTX_ENOMEM
    assert code(mtx.mtx_clip_grads, None, 1.0, None) == mtx.MTX_EINVAL
    mtx.mtx_free_clip(None)


def test_python_lists_of_tensors():
    import torch
    t = torch.zeros(6, 4)
    for pair in ((t.t(), None), (t.double(), None), (t, torch.zeros(23)), (t, torch.zeros(4, 6).t())):
        with pytest.raises(ValueError):
            mtx.make_tensor_list([pair])
    arr = mtx.make_tensor_list([(t, t), (torch.zeros(3, dtype=torch.bfloat16), torch.zeros(3))])
    assert arr[0].src == arr[0].dst and arr[1].src_type == B and arr[1].dst_type == F
    assert np.int64(arr[1].n) == 3


def test_token_networks():
    from paper_1704_04560_amd import workloads as wl

    def code_of(layers, shape=(1, 4, 1), dt=F, R=2):
        t = [(l.kind, l.out, l.k, l.stride, l.pad, l.groups, int(l.relu)) if isinstance(l, wl.Layer)
             else l for l in layers]
        with pytest.raises(mtx.MtxError) as e:
            mtx.mtx_model_sizes(mtx.make_desc(shape, t, dt), R, 2)
        return e.value.code

    ok = [wl.embed(10, 8), wl.norm(), wl.fc(3)]
    d = mtx.make_desc((1, 4, 1), [(l.kind, l.out, l.k, l.stride, l.pad, l.groups, 0) for l in ok], F)
    P, ld, ws = mtx.mtx_model_sizes(d, 2, 2)
    assert P == 10 * 8 + 2 * 8 + 3 * 32 + 3 and ld >= P and ws > 0
    for bad in ([wl.norm(), wl.embed(10, 8), wl.fc(3)], [wl.embed(0, 8), wl.fc(3)],
                [wl.embed(10, 0), wl.fc(3)], [(6, 8, 10, 1, 1, 1, 0), wl.fc(3)],
                [(6, 8, 10, 1, 0, 1, 1), wl.fc(3)], [(6, 8, 10, 2, 0, 1, 0), wl.fc(3)],
                [(6, 8, 10, 1, 0, 2, 0), wl.fc(3)], [wl.embed(10, 8), (7, 9, 0, 1, 0, 1, 0), wl.fc(3)],
                [wl.embed(10, 8), (7, 0, 2, 1, 0, 1, 0), wl.fc(3)],
                [wl.embed(10, 8), (7, 0, 1, 1, 0, 1, 1), wl.fc(3)],
                [wl.embed(10, 8), (7, 0, 1, 1, 2, 1, 0), wl.fc(3)], [wl.embed(10, 8), wl.norm()]):
        assert code_of(bad) == mtx.MTX_EINVAL, bad
    assert code_of(ok, shape=(2, 4, 1)) == mtx.MTX_EINVAL
    assert code_of(ok, R=65537) == mtx.MTX_EINVAL
    assert code_of([wl.embed(10, 16385), wl.norm(), wl.fc(3)]) == mtx.MTX_EUNSUPPORTED
    for f in (lambda: mtx.mtx_train_step_tokens(None, A[0], A[1], 0.1, 0.0, stream=0),
              lambda: mtx.mtx_set_embedding(None), lambda: mtx.mtx_set_clip_norm(None, 1.0)):
        with pytest.raises(mtx.MtxError):
            f()
