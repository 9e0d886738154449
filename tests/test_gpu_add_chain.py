"""Additions that follow one another (x + a + b): their steps against the oracle and, for token
networks, double-precision autograd.  Every addition but the last passes its output gradient on
unchanged, so all layers of such a chain read the gradient of its last sum."""
import pytest
import torch

from paper_1704_04560_amd import mtx
from paper_1704_04560_amd import workloads as wl
from tests import parity
from tests import test_gpu_token_step as tokens
from tests.test_gpu_train_step import run_case

pytestmark = pytest.mark.gpu

CHAINS = {
    "add add": (wl.conv(8, 3, pad=1, relu=True), wl.conv(8, 3, pad=1), wl.conv(8, 3, pad=1),
                wl.add(0), wl.add(1), wl.conv(6, 1), wl.fc(4)),
    "add add add": (wl.conv(8, 3, pad=1), wl.conv(8, 3, pad=1, relu=True), wl.conv(8, 1),
                    wl.conv(8, 3, pad=1), wl.add(0), wl.add(1), wl.add(2, relu=True), wl.fc(4)),
    "bn addp add add": (wl.conv(8, 3, pad=1), wl.bn(relu=True), wl.conv(8, 3, pad=1), wl.bn(),
                        wl.addp(1, 8), wl.add(0), wl.add(2), wl.conv(6, 1), wl.fc(4)),
    "add addp": (wl.conv(8, 3, pad=1, relu=True), wl.conv(8, 3, pad=1), wl.conv(8, 3, pad=1),
                 wl.add(0), wl.addp(1, 8, relu=True), wl.maxpool(2, 2), wl.fc(4)),
    # a ReLU between two additions, and a sum that a later addition reads
    "add relu, add": (wl.conv(8, 3, pad=1), wl.conv(8, 3, pad=1), wl.conv(8, 3, pad=1),
                      wl.add(0, relu=True), wl.add(1), wl.conv(8, 1), wl.add(4), wl.fc(4)),
}


@pytest.mark.parametrize("dtype", [wl.F32, wl.BF16])
@pytest.mark.parametrize("name", list(CHAINS))
def test_chain_of_additions(name, dtype, monkeypatch):
    # a bias before batch normalisation cancels only where no addition reads the layer as well
    cancels = parity.zero_by_batch_norm
    monkeypatch.setattr(parity, "zero_by_batch_norm", lambda geo, gi: cancels(geo, gi) and not any(
        l.kind in (wl.ADD, wl.ADDP) and l.k == gi for l in CHAINS[name]))
    net = wl.Net(name, (3, 8, 8), CHAINS[name], dtype, "normal")
    run_case(f"{name}-{dtype}", net, 2, 4, 2, seed=41, lr=0.01, mu=0.9)


TOKEN_CHAINS = {
    "add add norm": (wl.embed(61, 48), wl.conv(48, 1), wl.conv(48, 1), wl.add(0), wl.add(1),
                     wl.norm(), wl.fc(7)),
    "norm add add": (wl.embed(61, 48), wl.conv(48, 1, relu=True), wl.conv(48, 1), wl.norm(False),
                     wl.add(0), wl.add(2), wl.conv(48, 1), wl.fc(7)),
}


@pytest.mark.parametrize("dtype", [wl.F32, wl.BF16])
@pytest.mark.parametrize("name", list(TOKEN_CHAINS))
def test_chain_of_additions_over_tokens(name, dtype):
    net = wl.Net(name, (1, 9, 1), TOKEN_CHAINS[name], dtype, "normal")
    R, Nb = 2, 5
    print(f"[case] token chain {name} dtype={dtype}", flush=True)
    m = mtx.Model(net.in_shape, wl.layer_tuples(net), dtype, R, Nb, seed=2)
    tokens._spread(m, 3)
    w = torch.from_numpy(m.get_params()[0]).double()
    tok, lab = tokens._batch(net, R * Nb, 6)
    m.train_step(tok.cuda(), lab.cuda(), 0.05, 0.9)
    got = torch.from_numpy(m.grads_host()).double()
    for r in range(R):
        s = slice(r * Nb, (r + 1) * Nb)
        _, ref = tokens._ref_shard(net.layers, None, w, tok[s].long(), lab[s], dtype == wl.BF16,
                                   1.0, -1)
        off = 0
        for i, n in enumerate(tokens._param_sizes(net)):
            a, b = parity.rel_err(got[r, off:off + n].numpy(), ref[off:off + n].numpy())
            assert a <= parity.TOL[dtype], (i, r, a)
            if dtype == wl.F32:
                assert b <= parity.TOL[dtype], (i, r, b)
            off += n
    m.close()
