"""Norms and embeddings beside layers of images: a norm as the first layer, before and after pooling and
batch normalisation, an embedding that is pooled, batch-normalised, convolved over its neighbours or
read by the classifier at once.  fp32 steps against double-precision autograd."""
import numpy as np
import pytest
import torch
import torch.nn.functional as F

from paper_1704_04560_amd import mtx
from paper_1704_04560_amd import workloads as wl
from tests import parity

pytestmark = pytest.mark.gpu

NETS = {
    "norm first": ((3, 6, 5), (wl.norm(), wl.conv(8, 3, pad=1, relu=True), wl.fc(4))),
    "norm first, one channel": ((1, 6, 5), (wl.norm(), wl.conv(8, 3, pad=1), wl.fc(4))),
    "norm first, vectors": ((37, 1, 1), (wl.norm(False), wl.fc(12, relu=True), wl.norm(), wl.fc(4))),
    "conv norm pool": ((3, 8, 8), (wl.conv(12, 3, pad=1, relu=True), wl.norm(), wl.maxpool(2, 2),
                                   wl.conv(8, 3), wl.norm(False), wl.fc(4))),
    "pool norm fc": ((3, 8, 8), (wl.conv(12, 3, pad=1, relu=True), wl.maxpool(3, 2), wl.norm(False),
                                 wl.fc(4))),
    "norm pool fc": ((3, 8, 8), (wl.conv(12, 3, pad=1), wl.norm(), wl.maxpool(2, 2), wl.fc(4))),
    "bn add norm": ((3, 6, 6), (wl.conv(8, 3, pad=1, relu=True), wl.conv(8, 3, pad=1), wl.bn(),
                                wl.add(0), wl.norm(), wl.conv(8, 1), wl.bn(relu=True), wl.norm(False),
                                wl.fc(4))),
    "norm bn": ((3, 6, 6), (wl.conv(8, 3, pad=1, relu=True), wl.norm(False), wl.bn(), wl.fc(4))),
    "two norms": ((3, 5, 5), (wl.conv(20, 3, relu=True), wl.norm(), wl.norm(False), wl.fc(4))),
    "add relu norm": ((3, 6, 6), (wl.conv(8, 3, pad=1), wl.conv(8, 3, pad=1), wl.conv(8, 1),
                                  wl.add(0, relu=True), wl.norm(), wl.add(1), wl.norm(), wl.fc(4))),
    "embed fc": ((1, 4, 3), (wl.embed(30, 10), wl.fc(4))),
    "embed pool": ((1, 6, 4), (wl.embed(30, 10), wl.maxpool(2, 2), wl.norm(), wl.fc(4))),
    "embed bn": ((1, 6, 4), (wl.embed(30, 12), wl.bn(relu=True), wl.conv(8, 3, pad=1), wl.fc(4))),
    "embed conv 3": ((1, 6, 4), (wl.embed(30, 9), wl.conv(16, 3, pad=1, relu=True),
                                 wl.conv(9, 3, pad=1), wl.add(0), wl.norm(False), wl.fc(4))),
}


def _reference(layers, w, x, tok, lab):
    """(gradient, sizes of the parameter tensors, sums of |terms| of some) of one shard, NCHW, in double."""
    w, off, sizes, outs, a = w.clone().requires_grad_(True), 0, [], [], x
    scaled_away = {}   # a norm's weights before batch normalisation: parameter -> (output, hat)

    def take(*shape):
        nonlocal off
        n = int(np.prod(shape))
        sizes.append(n)
        off += n
        return w[off - n:off].view(*shape)

    def per_channel(t):
        return t[None, :, None, None]

    for i, l in enumerate(layers):
        if l.kind == wl.EMBED:
            a = take(l.k, l.out)[tok.long()].permute(0, 3, 1, 2)
        elif l.kind == wl.CONV:
            k, b = take(l.out, a.shape[1], l.k, l.k), take(l.out)
            a = F.conv2d(a, k, b, stride=l.stride, padding=l.pad)
        elif l.kind == wl.MAXPOOL:
            a = F.max_pool2d(a, l.k, l.stride)
        elif l.kind == wl.BN:
            g, b = take(a.shape[1]), take(a.shape[1])
            mean = a.mean((0, 2, 3), keepdim=True)
            var = (a - mean).square().mean((0, 2, 3), keepdim=True)
            a = (a - mean) / torch.sqrt(var + 1e-3) * per_channel(g) + per_channel(b)
        elif l.kind == wl.NORM:
            t = a - a.mean(1, keepdim=True) if l.k else a
            hat = t / torch.sqrt(t.square().mean(1, keepdim=True) + 1e-5)
            a = hat * per_channel(take(a.shape[1]))
            if layers[i + 1].kind == wl.BN:
                a.retain_grad()
                scaled_away[len(sizes) - 1] = a, hat.detach()
            a = a + per_channel(take(a.shape[1])) if l.k else a
        elif l.kind == wl.ADD:
            a = a + outs[l.k]
        elif l.kind == wl.FC:
            flat = a.reshape(a.shape[0], -1)
            k, b = take(l.out, flat.shape[1]), take(l.out)
            a = (flat @ k.t() + b)[:, :, None, None]
        a = torch.relu(a) if l.relu else a
        outs.append(a)
    F.cross_entropy(a[:, :, 0, 0], lab.long()).backward()
    assert off == w.numel()
    return w.grad, sizes, {k: (t.grad * hat).abs().sum((0, 2, 3)) for k, (t, hat) in scaled_away.items()}


@pytest.mark.parametrize("name", list(NETS))
def test_gradients(name):
    shape, layers = NETS[name]
    R, Nb = 2, 5
    print(f"[case] {name}", flush=True)
    net = wl.Net(name, shape, layers, wl.F32, "normal")
    m = mtx.Model(shape, wl.layer_tuples(net), wl.F32, R, Nb, seed=7)
    g = torch.Generator().manual_seed(len(name))
    w = torch.from_numpy(m.get_params()[0])
    w = w + 0.05 * torch.randn(w.shape, generator=g)
    m.set_params(w.numpy())
    x = torch.randn(R * Nb, *shape, generator=g)
    tok = torch.randint(0, 30, (R * Nb, *shape[1:]), generator=g, dtype=torch.int32)
    lab = torch.randint(0, 4, (R * Nb,), generator=g, dtype=torch.int32)
    tokens = layers[0].kind == wl.EMBED
    m.train_step(tok.cuda() if tokens else x.cuda(), lab.cuda(), 0.05, 0.9)
    got = torch.from_numpy(m.grads_host()).double()
    for r in range(R):
        s = slice(r * Nb, (r + 1) * Nb)
        ref, sizes, terms = _reference(layers, w.double(), x[s].double(), tok[s], lab[s])
        at, top = 0, float(ref.abs().max())
        for i, n in enumerate(sizes):
            a, b = got[r, at:at + n], ref[at:at + n]
            # a bias that batch normalisation removes again has no gradient: both hold rounding alone
            if float(b.abs().max()) < 1e-12 * top:
                assert float(a.abs().max()) <= parity.TOL[wl.F32] * top, (i, r)
            elif i in terms:
                # Batch normalisation takes a channel's scale out again, so the terms dy hat of the
                # weight's gradient cancel but for its eps.  Terms that are each within TOL of theirs
                # have sums that differ by at most TOL times the sum of their absolute values.
                assert bool(((a - b).abs() <= parity.TOL[wl.F32] * terms[i]).all()), (i, r)
            else:
                assert max(parity.rel_err(a.numpy(), b.numpy())) <= parity.TOL[wl.F32], (i, r)
            at += n
    m.close()
