"""Plain 64-bit forms of the token operators and the bounds on their fp32 evaluation.

A bound is U * K * (the same formula over absolute values) plus half a step of the output's type:
U = 2^-24 is half a step of fp32 relative to the value, K counts the roundings on the longest path
to an element (additions of a sum in any order, and the dozen or so operations around it), and the
formula over absolute values is what those relative errors act on where terms cancel.
"""
import torch

U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16


def half(dtype):
    """Half a step of a type, relative to the value."""
    return torch.finfo(dtype).eps / 2


def assert_within(got, ref, tol, what):
    got, ref, tol = got.double().cpu(), ref.double().cpu(), tol.double().cpu()
    bad = ~((got - ref).abs() <= tol)
    bad &= ~(torch.isnan(got) & torch.isnan(ref)) & ~(got == ref)
    if bad.any():
        at = tuple(int(v[0]) for v in torch.where(bad))
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {at}: got "
                             f"{got[at].item()!r}, want {ref[at].item()!r} +- {tol[at].item():.3g}")


def embed_grad(tok, dy, V, pad, scale):
    """(gradient [V][D], sum of |terms|, number of terms [V][1]) of one shard, in double."""
    tok, dy = tok.long().cpu(), dy.double().cpu()
    keep = (tok >= 0) & (tok < V) & ((tok != pad) if pad >= 0 else torch.ones_like(tok).bool())
    tok, dy = tok[keep], dy[keep] * scale
    z = torch.zeros(V, dy.shape[1], dtype=torch.float64)
    cnt = torch.zeros(V, dtype=torch.float64).index_add(0, tok, torch.ones(len(tok)).double())
    return z.index_add(0, tok, dy), z.index_add(0, tok, dy.abs()), cnt[:, None]


class Norm:
    """Forward and backward of the block norm in double, with bounds.  Parameters are dicts of CPU
    double tensors (None where absent)."""

    def __init__(self, layer, eps, scale, group, p, R):
        self.layer, self.eps, self.scale, self.group, self.p, self.R = layer, eps, scale, group, p, R

    def gate_rows(self, rows):
        g = self.p["gate"]
        if g is None:
            return 1.0
        return g.repeat_interleave(self.group, 0) if self.group else g.reshape(1, -1)

    def _norm(self, t, m, w, b):
        """(norm, its magnitude, mean, r, spread) of rows t with magnitude m."""
        mean = t.mean(1, keepdim=True) if self.layer else torch.zeros(len(t), 1).double()
        mm = m + (m.mean(1, keepdim=True) if self.layer else 0.0)
        r = ((t - mean).square().mean(1, keepdim=True) + self.eps).rsqrt()
        # the relative error of r is that of the mean square over itself
        spread = mm.square().mean(1, keepdim=True) * r * r
        y = (t - mean) * r * w
        my = mm * r * w.abs() + y.abs() * spread
        if b is not None:
            y, my = y + b, my + b.abs()
        return y, my, mean, r, spread

    def forward(self, h, x):
        p = self.p
        st = torch.zeros(len(h), 4).double()
        mst = torch.zeros(len(h), 4).double()
        H, mH = h, h.abs()
        if x is not None:
            u, mu = x, x.abs()
            if p["post_w"] is not None:
                u, mu, mean, r, sp = self._norm(x, x.abs(), p["post_w"], p["post_b"])
                st[:, 0:1], st[:, 1:2] = mean, r
                mst[:, 0:1], mst[:, 1:2] = x.abs().mean(1, keepdim=True), r * (1 + sp)
            g = self.gate_rows(len(h))
            H = h + self.scale * g * u
            mH = h.abs() + abs(self.scale) * (g if isinstance(g, float) else g.abs()) * mu
        y = my = None
        if p["pre_w"] is not None:
            y, my, mean, r, sp = self._norm(H, mH, p["pre_w"], p["pre_b"])
            st[:, 2:3], st[:, 3:4] = mean, r
            mst[:, 2:3], mst[:, 3:4] = mH.mean(1, keepdim=True), r * (1 + sp)
        return dict(h=H, y=y, st=st), dict(h=mH, y=my, st=mst)

    def _pull(self, g, mg, hat, mhat, r):
        out = g - hat * (g * hat).mean(1, keepdim=True)
        mag = mg + mhat * (mg * mhat).mean(1, keepdim=True)
        if self.layer:
            out, mag = out - g.mean(1, keepdim=True), mag + mg.mean(1, keepdim=True)
        return out * r, mag * r

    def backward(self, H, x, st, dy, dho):
        """Gradients and magnitudes from the statistics that the forward pass kept."""
        p, R = self.p, self.R
        N, D = (dy if dy is not None else dho).shape
        v, m = {}, {}

        def shard(name, a, ma, group=None):
            k = (N // group) if group else R
            v[name] = a.reshape(k, N // k, D).sum(1) if N else torch.zeros(k, D).double()
            m[name] = ma.reshape(k, N // k, D).sum(1) if N else torch.zeros(k, D).double()

        dH = dho if dho is not None else torch.zeros(N, D).double()
        mH = dH.abs()
        if dy is not None:
            mean, r = st[:, 2:3], st[:, 3:4]
            hat, mhat = (H - mean) * r, (H.abs() + mean.abs()) * r
            shard("pre_w", dy * hat, dy.abs() * mhat)
            shard("pre_b", dy, dy.abs())
            g, mg = self._pull(dy * p["pre_w"], (dy * p["pre_w"]).abs(), hat, mhat, r)
            dH, mH = dH + g, mH + mg
        v["dh"], m["dh"] = dH, mH
        if x is None:
            return v, m
        g = self.gate_rows(N)
        ag = g if isinstance(g, float) else g.abs()
        du, mdu = self.scale * g * dH, abs(self.scale) * ag * mH
        u, mu = x, x.abs()
        v["dx"], m["dx"] = du, mdu
        if p["post_w"] is not None:
            mean, r = st[:, 0:1], st[:, 1:2]
            hat, mhat = (x - mean) * r, (x.abs() + mean.abs()) * r
            shard("post_w", du * hat, mdu * mhat)
            shard("post_b", du, mdu)
            u, mu = hat * p["post_w"], mhat * p["post_w"].abs()
            if p["post_b"] is not None:
                u, mu = u + p["post_b"], mu + p["post_b"].abs()
            v["dx"], m["dx"] = self._pull(du * p["post_w"], mdu * p["post_w"].abs(), hat, mhat, r)
        shard("gate", self.scale * dH * u, abs(self.scale) * mH * mu, self.group or None)
        return v, m
