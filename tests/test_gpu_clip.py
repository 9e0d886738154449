"""Global gradient norm and clipping on the GPU against 64-bit forms, through the C ABI."""
import pytest
import torch

from paper_1704_04560_amd import mtx
from tests.ops_ref import BF16, F32, U, assert_within, half

pytestmark = pytest.mark.gpu


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _ws():
    return torch.empty(mtx.MTX_CLIP_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("ratio", [0.3, 0.999, 1.5, float("inf")])
@pytest.mark.parametrize("R,n,ld,off", [
    (1, 1, 1, 0), (2, 3, 9, 1), (4, 255, 256, 0), (3, 1000, 1003, 0), (8, 4099, 4100, 0),
    (16, 70001, 70016, 0), (1, 300000, 300000, 0), (2, 203530, 203584, 0), (5, 2_000_003, 2_000_004, 3)])
def test_average_clip(R, n, ld, off, ratio):
    """Element: R - 1 additions and a division, then one product; norm: the elements' errors, and
    one rounding (the squares are added in double)."""
    print(f"[case] average_clip R={R} n={n} ld={ld} off={off} ratio={ratio}", flush=True)
    g = _gen(R + n)
    buf = torch.randn(R * ld + off, generator=g) * 0.01
    rows = buf[off:].view(R, ld)[:, :n].double()
    ref, mag = rows.mean(0), rows.abs().mean(0)
    norm = float(ref.norm())
    max_norm = ratio * norm if norm else ratio
    dev = buf.cuda()
    out = torch.full((n + 8 + off,), 7.0, device="cuda")
    avg, nrm = out[off:off + n], torch.full((1,), -1.0, device="cuda")
    mtx.mtx_average_clip(dev[off:], R, n, ld, max_norm, avg, nrm, _ws())
    torch.cuda.synchronize()
    err = U * (R + 1) * mag
    dn = float(err.norm())
    assert_within(nrm, torch.tensor([norm]), torch.tensor([dn + U * norm * 2]), "norm")
    f = min(1.0, ratio)
    assert_within(avg, ref * f, f * (err + ref.abs() * (dn / max(norm, 1e-300) + 4 * U)), "average")
    assert (out[:off] == 7.0).all() and (out[off + n:] == 7.0).all()
    if ratio > 1:   # unclipped: the plain average's bits
        plain = torch.empty(n, device="cuda")
        mtx.mtx_average_grads(dev[off:], R, n, ld, plain)
        assert torch.equal(plain, avg)
    again = torch.empty(n, device="cuda")
    mtx.mtx_average_clip(dev[off:], R, n, ld, max_norm, again, None, _ws())
    if off % 4 == 0:
        assert torch.equal(again, avg)


def _sizes(count, g):
    s = [0, 1, 7, 16384, 16385, 3, 40000, 8, 2, 100003]
    return (s * (count // len(s) + 1))[:count]


@pytest.mark.parametrize("st", [F32, BF16])
@pytest.mark.parametrize("dt", [F32, BF16, "in place", None])
@pytest.mark.parametrize("count,ratio,shift", [(1, 0.5, 0), (3, 0.5, 1), (10, 0.7, 0), (10, 2.0, 3),
                                               (301, 0.01, 1), (37, float("inf"), 0)])
def test_clip_list(count, ratio, shift, st, dt):
    """Tensors at odd offsets of one allocation; what lies between them stays."""
    print(f"[case] clip_list count={count} ratio={ratio} shift={shift} {st} -> {dt}", flush=True)
    g = _gen(count)
    sizes = _sizes(count, g)
    if not any(sizes):
        sizes = [5]
    src, dst, ref = [], [], []
    total = sum(n + shift for n in sizes) + 8
    a = torch.full((total,), 3.0, dtype=st, device="cuda")
    b = torch.full((total,), 3.0, dtype=dt if dt in (F32, BF16) else F32, device="cuda")
    o = shift
    for n in sizes:
        a[o:o + n] = (torch.randn(n, generator=g) * 0.01).to(st).cuda()
        src.append(a[o:o + n])
        ref.append(a[o:o + n].double().cpu())
        dst.append(src[-1] if dt == "in place" else None if dt is None else b[o:o + n])
        o += n + shift
    flat = torch.cat(ref)
    norm = float(flat.norm())
    before = a.clone()
    clip = mtx.Clip(list(zip(src, dst)))
    nrm = torch.empty(1, device="cuda")
    clip.clip(ratio * norm, nrm)
    torch.cuda.synchronize()
    assert_within(nrm, torch.tensor([norm]), torch.tensor([2 * U * norm]), "norm")
    if dt != "in place":
        assert torch.equal(a.view(torch.uint8), before.view(torch.uint8))
    if dt is None:
        return
    f = min(1.0, ratio)
    t = dst[0].dtype
    for i, (d, r) in enumerate(zip(dst, ref)):
        assert_within(d, f * r, f * r.abs() * (half(t) + 4 * U), f"tensor {i}")
    whole = b if dt != "in place" else a
    mask = torch.ones(total, dtype=torch.bool)
    o = shift
    for n in sizes:
        mask[o:o + n] = False
        o += n + shift
    assert (whole.cpu()[mask] == 3.0).all()
    if f == 1.0 and dt in (st, "in place"):
        assert torch.equal(whole.cpu()[~mask], before.cpu()[~mask])
    clip.close()


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_a_norm_that_is_not_finite_clips_nothing(bad):
    g = torch.randn(5000, generator=_gen(1))
    g[77] = bad
    a, out = g.cuda(), torch.empty(5000, device="cuda")
    nrm = torch.zeros(1, device="cuda")
    clip = mtx.Clip([(a, out)])
    clip.clip(0.1, nrm)
    torch.cuda.synchronize()
    assert not torch.isfinite(nrm).item()
    assert torch.equal(out.cpu().view(torch.int32), g.view(torch.int32))
    avg = torch.empty(5000, device="cuda")
    mtx.mtx_average_clip(a, 1, 5000, 5000, 0.1, avg, nrm, _ws())
    assert not torch.isfinite(nrm).item()
    keep = torch.isfinite(g)
    assert torch.equal(avg.cpu()[keep], g[keep])


def test_large_and_tiny_values():
    """Squares beyond fp32's range on both sides still give the norm."""
    for v, m in ((3e30, 1.0), (1e-30, 1.0), (3e33, 1e-20)):   # (a factor below fp32's range)
        a = torch.full((1000,), v, device="cuda")
        nrm = torch.zeros(1, device="cuda")
        avg = torch.empty(1000, device="cuda")
        mtx.mtx_average_clip(a, 1, 1000, 1000, m, avg, nrm, _ws())
        clip = mtx.Clip([(a, a)])
        clip.clip(m, nrm)
        torch.cuda.synchronize()
        x = float(torch.tensor(v, dtype=F32).double())
        want = x * 1000 ** 0.5
        assert abs(nrm.item() - want) <= 2 * U * want
        ref = min(1.0, float(torch.tensor(m).double()) / want) * x
        assert abs(a[0].item() - ref) <= 4 * U * ref and torch.equal(a, avg)


def test_zero_gradients():
    a = torch.zeros(300, device="cuda")
    nrm = torch.ones(1, device="cuda")
    mtx.Clip([(a, a)]).clip(0.5, nrm)
    assert nrm.item() == 0.0 and not a.any()


def test_captured_and_replayed():
    """Two graphs with workspaces of their own, replayed with new gradients."""
    g = _gen(4)
    n = 100_000
    a, out, nrm = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty(2, device="cuda")
    rows, avg = torch.empty(3, n, device="cuda"), torch.empty(n, device="cuda")
    clip, ws = mtx.Clip([(a, out)]), _ws()
    a.fill_(1.0), rows.fill_(1.0)
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    torch.cuda.synchronize()
    with torch.cuda.graph(graphs[0]):
        clip.clip(0.5, nrm)
    with torch.cuda.graph(graphs[1]):
        mtx.mtx_average_clip(rows, 3, n, n, 0.5, avg, nrm[1:], ws)
    for k in range(3):
        a.copy_(torch.randn(n, generator=g) * 10 ** -k)
        rows.copy_(torch.randn(3, n, generator=g))
        clip.clip(0.5, nrm)
        mtx.mtx_average_clip(rows, 3, n, n, 0.5, avg, nrm[1:], ws)
        want = [t.clone() for t in (out, avg, nrm)]
        for t in (out, avg, nrm):
            t.zero_()
        graphs[1].replay()
        graphs[0].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(want, (out, avg, nrm)))


def test_norm_out_inside_the_list_is_refused():
    a = torch.ones(300, device="cuda")
    b = torch.ones(300, device="cuda")
    clip = mtx.Clip([(a[:100], None), (a[50:200], None), (b, b)])
    for bad in (a[0:], a[199:], b[299:], b[150:], clip.workspace[64:]):
        with pytest.raises(mtx.MtxError) as e:
            clip.clip(1.0, bad)
        assert e.value.code == mtx.MTX_EINVAL
    clip.clip(1.0, a[200:])
    assert abs(a[200].item() - 550 ** 0.5) <= 2 * U * 550 ** 0.5


def test_two_graphs_of_one_handle_and_workspace():
    """Replayed in turn, each with its own bound, over workspaces that they share."""
    g = _gen(6)
    n = 50_001
    a, out, nrm = torch.zeros(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty(1, device="cuda")
    rows, avg = torch.zeros(2, n, device="cuda"), torch.empty(n, device="cuda")
    clip, ws = mtx.Clip([(a, out)]), _ws()
    graphs = []
    torch.cuda.synchronize()
    for m in (0.5, 2.0):
        graphs.append((m, torch.cuda.CUDAGraph()))
        with torch.cuda.graph(graphs[-1][1]):
            clip.clip(m, nrm)
            mtx.mtx_average_clip(rows, 2, n, n, m, avg, None, ws)
    for k in range(4):
        a.copy_(torch.randn(n, generator=g))
        rows.copy_(torch.randn(2, n, generator=g))
        m, graph = graphs[k % 2]
        clip.clip(m, nrm)
        mtx.mtx_average_clip(rows, 2, n, n, m, avg, None, ws)
        want = [t.clone() for t in (out, avg, nrm)]
        for t in (out, avg, nrm):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(want, (out, avg, nrm)))
