"""Training steps of token networks without clipping: the execution options give the same bits, and
projection shortcuts from an embedding and from a norm match double-precision autograd."""
import numpy as np
import pytest
import torch
import torch.nn.functional as F

from paper_1704_04560_amd import mtx
from paper_1704_04560_amd import workloads as wl
from tests import parity
from tests import test_gpu_token_step as tokens

pytestmark = pytest.mark.gpu

WIDE = wl.Net("wide", (1, 8, 1), (wl.embed(300, 512), wl.norm(False), wl.fc(2048, relu=True), wl.norm(),
                                  wl.fc(10)), wl.F32, "normal")
OPTIONS = {"layerwise": (mtx.mtx_set_layerwise_update,), "overlap": (mtx.mtx_set_overlap,),
           "overlap and layerwise": (mtx.mtx_set_overlap, mtx.mtx_set_layerwise_update),
           "graph": (mtx.mtx_set_graph_replay,), "timing": (mtx.mtx_set_timing,),
           "graph of three streams": (mtx.mtx_set_overlap, mtx.mtx_set_layerwise_update,
                                      mtx.mtx_set_graph_replay),
           "check": (mtx.mtx_set_nonfinite_check,)}


@pytest.mark.parametrize("dtype", [wl.F32, wl.BF16])
@pytest.mark.parametrize("rule", [mtx.MTX_OPT_MOMENTUM, mtx.MTX_OPT_ADAM])
@pytest.mark.parametrize("name", ["res", "odd", "bag", "wide"])
def test_options_give_the_same_bits(name, rule, dtype):
    net = tokens._net(name, dtype) if name != "wide" else wl.Net("wide", WIDE.in_shape, WIDE.layers,
                                                                 dtype, "normal")
    print(f"[case] token options {name} rule={rule} dtype={dtype}", flush=True)
    R, Nb = 2, 8
    batches = [tuple(t.cuda() for t in tokens._batch(net, R * Nb, k)) for k in range(2)]
    tok, lab = (torch.empty_like(t) for t in batches[0])

    def run(setters):
        m = tokens._model(net, R, Nb, seed=3)
        mtx.mtx_set_embedding(m.handle, 2.0, 1)
        m.set_optimizer(rule)
        mtx.mtx_set_overlap(m.handle, False)
        if setters is None:
            mtx.mtx_set_fused_update(m.handle, False)
        for f in setters or ():
            f(m.handle, True)
        for k in range(4):
            tok.copy_(batches[k % 2][0])
            lab.copy_(batches[k % 2][1])
            m.train_step(tok, lab, 0.02, 0.9)
        torch.cuda.synchronize()
        got = [*m.get_params(), m.grads_host(), m.grad_avg.cpu().numpy()]
        fused = [l["layer"] for l in mtx.mtx_get_launches(m.handle)
                 if l["flags"] & mtx.MTX_GEMM_FUSED_UPDATE]
        m.close()
        return got, fused

    want, none = run(None)   # one stream, one average and update at the end
    assert not none
    plain, fused = run(())
    assert bool(fused) == (name == "wide" and rule == mtx.MTX_OPT_MOMENTUM)
    for a, b in zip(plain, want):
        assert np.array_equal(a.view(np.uint32), b.view(np.uint32)), "fused"
    for option, setters in OPTIONS.items():
        if option == "check" and rule != mtx.MTX_OPT_MOMENTUM:
            continue
        got, _ = run(setters)
        for a, b in zip(got, want):
            assert np.array_equal(a.view(np.uint32), b.view(np.uint32)), option


@pytest.mark.parametrize("R,Nb", [(1, 6), (3, 4)])
def test_projections_from_an_embedding_and_a_norm(R, Nb):
    V, C, T = 40, 32, 6
    layers = (wl.embed(V, C), wl.conv(24, 1, relu=True), wl.conv(16, 1), wl.addp(0, 16), wl.norm(),
              wl.conv(C, 1, relu=True), wl.conv(20, 1), wl.addp(4, 20), wl.norm(False), wl.fc(5))
    net = wl.Net("projections", (1, T, 1), layers, wl.F32, "normal")
    print(f"[case] token projections R={R} Nb={Nb}", flush=True)
    m = tokens._model(net, R, Nb, seed=4)
    tokens._spread(m, 5)
    w0 = torch.from_numpy(m.get_params()[0]).double()
    tok, lab = tokens._batch(net, R * Nb, 2)
    m.train_step(tok.cuda(), lab.cuda(), 0.05, 0.9)
    got = torch.from_numpy(m.grads_host()).double()
    for r in range(R):
        s = slice(r * Nb, (r + 1) * Nb)
        w, off, sizes = w0.clone().requires_grad_(True), 0, []

        def take(*shape):
            nonlocal off
            n = int(np.prod(shape))
            sizes.append(n)
            off += n
            return w[off - n:off].view(*shape)

        def conv(a, out):
            k, b = take(out, a.shape[-1]), take(out)
            return a @ k.t() + b

        def norm(a, layer):
            a = a - a.mean(-1, keepdim=True) if layer else a
            a = a / torch.sqrt(a.square().mean(-1, keepdim=True) + 1e-5) * take(a.shape[-1])
            return a + take(a.shape[-1]) if layer else a

        e = take(V, C)[tok[s].long()]
        a = conv(torch.relu(conv(e, 24)), 16)
        n = norm(a + conv(e, 16), True)
        a = conv(torch.relu(conv(n, C)), 20)
        a = norm(a + conv(n, 20), False)
        x = a.transpose(1, 2).reshape(Nb, -1)   # channels, then positions
        k, b = take(5, x.shape[1]), take(5)
        F.cross_entropy(x @ k.t() + b, lab[s].long()).backward()
        assert off == w.numel()
        at = 0
        for i, size in enumerate(sizes):
            rel = parity.rel_err(got[r, at:at + size].numpy(), w.grad[at:at + size].numpy())
            assert max(rel) <= parity.TOL[wl.F32], (i, r, rel)
            at += size
    m.close()


@pytest.mark.parametrize("dtype", [wl.F32, wl.BF16])
def test_stored_outputs_of_the_token_layers(dtype):
    """The embedding's rows bit for bit, and each norm from the stored outputs before it: fp32 sums of
    24 terms and a dozen operations around them, and the rounding of what is stored."""
    C, T, R, Nb = 24, 10, 2, 3
    net = wl.Net("outputs", (1, 5, 2), (wl.embed(50, C), wl.norm(), wl.conv(C, 1), wl.norm(False),
                                        wl.add(0), wl.norm(), wl.fc(3)), dtype, "normal")
    m = tokens._model(net, R, Nb, seed=6)
    mtx.mtx_set_embedding(m.handle, 5.0, 7)
    tokens._spread(m, 2)
    w = m.get_params()[0]
    tok, lab = tokens._batch(net, R * Nb, 4)
    tok[0, 3] = 7
    m.train_step(tok.cuda(), lab.cuda(), 0.01, 0.9)
    out = [torch.from_numpy(m.layer_output(i)).view(R * Nb, -1, T) for i in range(6)]
    table = torch.from_numpy(w[:50 * C]).view(50, C)
    rows = table[tok.long()] * 5.0
    rows[tok == 7] = 0.0
    want = (rows.bfloat16().float() if dtype == wl.BF16 else rows).transpose(1, 2)
    assert torch.equal(out[0], want)
    step = 2.0 ** -8 if dtype == wl.BF16 else 0.0
    total = out[0].double() + out[3].double()
    assert ((out[4].double() - total).abs() <= (step + 2.0 ** -24) * total.abs()).all()
    where = np.cumsum([0] + tokens._param_sizes(net))
    for i, src, p, layer in ((1, out[0].double(), 1, True), (3, out[2].double(), 5, False),
                             (5, total, 6, True)):
        a = src - src.mean(1, keepdim=True) if layer else src
        r = 1 / torch.sqrt(a.square().mean(1, keepdim=True) + 1e-5)
        g = torch.from_numpy(w[where[p]:where[p] + C]).double()[:, None]
        y = a * r * g
        if layer:
            y = y + torch.from_numpy(w[where[p + 1]:where[p + 1] + C]).double()[:, None]
        # fp32: sums of 24 terms and a dozen operations on values of the row's size
        scale = (src.abs() + src.abs().mean(1, keepdim=True)) * r * g.abs() + y.abs()
        cond = src.square().mean(1, keepdim=True) * r * r
        tol = step * y.abs() + 64 * 2.0 ** -24 * scale * (1 + cond)
        assert ((out[i].double() - y).abs() <= tol).all(), i
    m.close()
