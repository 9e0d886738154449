"""Operators of language-model training, as cases that can be timed and compared.

A case is a dict of plain values; `op` names the operator:
  embed_fwd   rows of an embedding table looked up by token and scaled
  embed_bwd   the table's gradient, one per shard, dense or added to what is there
  norm_fwd    residual addition of a block's output (normalised, gated, scaled) and the next norm
  norm_bwd    its gradients: stream, block output, norm weights and gate, the weights' per shard
  clip_list   global norm over many tensors, and their clipped fp32 copies in one flat vector
  clip_avg    average of R shard gradient rows with its global norm, clipped

With `own` false, run() computes them from elementary torch operations.  Token frequencies fall
as 1 / rank, as in text, with a share of padding where a case has it.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


def _embed(name, op, V, D, n, R=1, dtype="bf16", table="f32", pad=-1, padded=0.0, scale=1.0,
           accumulate=False):
    return {"name": name, "op": op, "V": V, "D": D, "n": n, "R": R, "dtype": dtype,
            "table": table, "pad": pad, "padded": padded, "scale": scale,
            "accumulate": accumulate}


def _norm(name, op, rows, D, R=1, dtype="bf16", layer=False, post=True, gate=True, group=0,
          scale=1.0):
    return {"name": name, "op": op, "rows": rows, "D": D, "R": R, "dtype": dtype, "layer": layer,
            "post": post, "gate": gate, "group": group, "scale": scale}


def _list(name, count, largest, dtype, clipped):
    return {"name": name, "op": "clip_list", "count": count, "largest": largest, "dtype": dtype,
            "clipped": clipped}


def _avg(name, R, n, ld, clipped):
    return {"name": name, "op": "clip_avg", "R": R, "n": n, "ld": ld, "clipped": clipped}


def listed():
    return [
        # Eight sequences, one new token each: latency.
        _embed("embed_fwd_tokens", "embed_fwd", 32768, 2048, 8, table="bf16", scale=1.0),
        # The lookup of a large training step from the fp32 master table, scaled by sqrt(D).
        _embed("embed_fwd_train", "embed_fwd", 131072, 4096, 32768, scale=64.0),
        # A small text classifier's table: odd sizes, fp32, four shards, padded sentences.
        _embed("embed_bwd_small", "embed_bwd", 5003, 300, 257, R=4, dtype="f32", pad=0, padded=0.3),
        # The dense gradient of a large table from one shard of 32768 tokens.
        _embed("embed_bwd_train", "embed_bwd", 131072, 2048, 32768, scale=45.25),
        # A table tied to the class scores: their gradient is in the rows already, two shards.
        _embed("embed_bwd_tied", "embed_bwd", 50001, 1024, 16383, R=2, accumulate=True),
        # The residual stream of eight new tokens through post-norm, addition and next pre-norm.
        _norm("norm_fwd_tokens", "norm_fwd", 8, 4096, gate=False),
        # The same of a training step, with a learned gate on the block's output.
        _norm("norm_fwd_train", "norm_fwd", 16384, 4096, scale=0.5),
        # ... and its backward pass over four shards.
        _norm("norm_bwd_train", "norm_bwd", 8192, 4096, R=4, scale=0.5),
        # Layer norm after an addition in fp32, odd sizes, a gate per sequence of 59 rows.
        _norm("norm_bwd_ragged", "norm_bwd", 8850, 771, R=3, dtype="f32", layer=True, post=False,
              group=59),
        # Two replicas' gradients of a 784-256-10 MLP averaged and clipped: latency.
        _avg("clip_avg_mlp", 2, 203_530, 203_584, True),
        # bf16 gradients of a few hundred tensors of mixed sizes into the flat fp32 row that the
        # update rules read.
        _list("clip_list_bf16", 291, 2_097_152, "bf16", True),
        # Sixteen replicas' gradients of 61 million parameters, averaged and clipped.
        _avg("clip_avg_61m", 16, 61_000_000, 61_000_000, True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    case = _draw(rng)
    del case["name"]
    return case


def _draw(rng):
    op = rng.choice(["embed_fwd", "embed_bwd", "norm_fwd", "norm_bwd", "clip_list", "clip_avg"])
    if op.startswith("embed"):
        D = _log(rng, 64, 4096)
        V = _log(rng, 1000, 131072)
        R = rng.choice([1, 1, 2, 4]) if op == "embed_bwd" else 1
        while op == "embed_bwd" and R * V * D > 131072 * 2048:
            V = max(1000, V // 2)
            R = max(1, R // 2)
        n = _log(rng, 1, 32768) // R + 1
        pad = rng.choice([-1, 0])
        return _embed("", op, V, D, n, R, rng.choice(["bf16", "f32"]), rng.choice(["bf16", "f32"]),
                      pad, rng.choice([0.1, 0.5]) if pad >= 0 else 0.0,
                      rng.choice([1.0, math.sqrt(D)]),
                      op == "embed_bwd" and rng.random() < 0.4)
    if op.startswith("norm"):
        D = _log(rng, 64, 8192)
        R = rng.choice([1, 2, 4]) if op == "norm_bwd" else 1
        group = rng.choice([0, 0, _log(rng, 1, 512)])
        most = (8192 if op == "norm_bwd" else 16384) * 4096 // D
        rows = _log(rng, 1, min(most, 65536))
        unit = R * max(1, group)
        rows = max(1, rows // unit) * unit
        post = rng.random() < 0.6
        return _norm("", op, rows, D, R, rng.choice(["bf16", "f32"]), rng.random() < 0.4, post,
                     rng.random() < 0.6 or group > 0, group, rng.choice([1.0, 0.5]))
    if op == "clip_list":
        return _list("", _log(rng, 1, 400), _log(rng, 1000, 1_000_000),
                     rng.choice(["bf16", "f32"]), rng.random() < 0.7)
    R = rng.choice([1, 2, 3, 4, 8, 16])
    n = _log(rng, 1000, 61_000_000)
    return _avg("", R, n, n + rng.choice([0, 0, 5, 64]), rng.random() < 0.7)


def _sizes(case, seed):
    """Lengths of a list's tensors: spread over their logarithm up to the largest, odd ones too."""
    g = torch.Generator().manual_seed(seed)
    u = torch.rand(case["count"], generator=g, dtype=torch.float64)
    return [max(1, int(v)) for v in (case["largest"] ** (0.25 + 0.75 * u)).tolist()]


def _tokens(case, g, n):
    V = case["V"]
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    rank = (torch.exp(u * math.log(V)) - 1.0).long().clamp_(0, V - 1)   # p(rank) ~ 1 / rank
    t = (rank * 7919 + 1) % V if V % 7919 else rank
    if case["pad"] >= 0:
        drop = torch.rand(n, generator=g, device="cuda") < case["padded"]
        t = torch.where(drop, torch.full_like(t, case["pad"]), t)
    return t.to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]

    def rand(*shape, dtype=torch.float32, mean=0.0, std=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * std + mean).to(dtype)

    s = {"case": case}
    if own:
        from paper_1704_04560_amd import mtx
        s["mtx"] = mtx
    if op.startswith("embed"):
        V, D, R, n = case["V"], case["D"], case["R"], case["n"]
        s["tokens"] = _tokens(case, g, R * n)
        if op == "embed_fwd":
            s["w"] = rand(V, D, dtype=TYPES[case["table"]], std=0.02)
            s["y"] = torch.empty(R * n, D, device="cuda", dtype=TYPES[case["dtype"]])
        else:
            s["dy"] = rand(R * n, D, dtype=TYPES[case["dtype"]], std=0.01)
            s["grads"] = (rand(R, V * D, std=0.01) if case["accumulate"]
                          else torch.empty(R, V * D, device="cuda"))
            if own:
                size = s["mtx"].mtx_embed_sizes(n, R, V, D)
                s["ws"] = torch.empty(size, device="cuda", dtype=torch.uint8)
    elif op.startswith("norm"):
        N, D, R, dt = case["rows"], case["D"], case["R"], TYPES[case["dtype"]]
        # a residual stream: a few channels are far larger than the rest
        wide = 1.0 + 20.0 * (torch.rand(D, generator=g, device="cuda") < 0.01)
        s["h"] = (rand(N, D) * wide).to(dt)
        s["x"] = rand(N, D, dtype=dt, std=0.7, mean=0.05)
        s["pre_w"] = rand(D, mean=1.0, std=0.1)
        s["pre_b"] = rand(D, std=0.1) if case["layer"] else None
        s["post_w"] = rand(D, mean=1.0, std=0.1) if case["post"] else None
        s["post_b"] = rand(D, std=0.1) if case["post"] and case["layer"] else None
        G = 1 if not case["group"] else N // case["group"]
        s["gate"] = rand(G, D, mean=0.3, std=0.2) if case["gate"] else None
        if op == "norm_fwd":
            s["h_out"], s["y"] = torch.empty_like(s["h"]), torch.empty_like(s["h"])
            s["stats"] = torch.empty(N, 4, device="cuda")
        else:
            s["dy"] = rand(N, D, dtype=dt, std=0.01)
            s["dh_out"] = rand(N, D, dtype=dt, std=0.01)
            s["stats"] = torch.zeros(N, 4, device="cuda")   # what the forward pass kept
            for col, t in ((0, s["x"]), (2, s["h"])):
                t = t.double()
                mean = t.mean(1) if case["layer"] else torch.zeros(N, device="cuda").double()
                s["stats"][:, col] = mean.float()
                var = (t - mean[:, None]).square().mean(1)
                s["stats"][:, col + 1] = (var + EPS).rsqrt().float()
            s["dh"], s["dx"] = torch.empty_like(s["h"]), torch.empty_like(s["h"])
            s["ld"] = 5 * D + 3 * (D % 2)       # the shards' gradient rows
            s["grads"] = torch.zeros(R, s["ld"], device="cuda")
            s["dgate"] = torch.empty(G, D, device="cuda") if case["group"] else None
        if own:
            mtx = s["mtx"]
            s["desc"] = mtx.make_norm_desc(
                mtx.MTX_NORM_LAYER if case["layer"] else mtx.MTX_NORM_RMS,
                mtx.MTX_BF16 if case["dtype"] == "bf16" else mtx.MTX_F32, N, D, EPS, case["scale"],
                case["group"], s["post_w"], s["post_b"], s["gate"], s["pre_w"], s["pre_b"])
            if op == "norm_bwd":
                size = mtx.mtx_block_norm_sizes(s["desc"], R)
                s["ws"] = torch.empty(size, device="cuda", dtype=torch.uint8)
    elif op == "clip_list":
        sizes = _sizes(case, 11)
        flat = rand(sum(sizes), std=0.01)
        s["src"] = [t.to(TYPES[case["dtype"]]) for t in flat.split(sizes)]
        s["dst"] = torch.empty_like(flat)
        s["max_norm"] = 0.01 * math.sqrt(flat.numel()) * (0.5 if case["clipped"] else 2.0)
        if own:
            s["norm"] = torch.empty(1, device="cuda")
            s["clip"] = s["mtx"].Clip(list(zip(s["src"], s["dst"].split(sizes))))
    else:
        R, n, ld = case["R"], case["n"], case["ld"]
        s["grads"] = rand(R, ld, std=0.01)
        s["avg"], s["norm"] = torch.empty(n, device="cuda"), torch.empty(1, device="cuda")
        s["max_norm"] = 0.01 * math.sqrt(n / R) * (0.5 if case["clipped"] else 2.0)
        if own:
            size = s["mtx"].MTX_CLIP_WORKSPACE_BYTES
            s["ws"] = torch.empty(size, device="cuda", dtype=torch.uint8)
    return s


def run(s):
    case = s["case"]
    return (_run_own if own else _run_plain)[case["op"]](s, case)


# ---- the framework's operators ------------------------------------------------------------------

def _mt(s, name):
    return s["mtx"].MTX_BF16 if name == "bf16" else s["mtx"].MTX_F32


def _own_embed_fwd(s, c):
    s["mtx"].mtx_embed_forward(s["w"], _mt(s, c["table"]), c["V"], c["D"], s["tokens"], c["n"],
                               c["pad"], c["scale"], s["y"], _mt(s, c["dtype"]), c["D"])
    return s["y"]


def _own_embed_bwd(s, c):
    s["mtx"].mtx_embed_backward(s["tokens"], c["n"], c["R"], s["dy"], _mt(s, c["dtype"]), c["D"],
                                c["V"], c["D"], c["pad"], c["scale"], s["grads"],
                                c["V"] * c["D"], c["accumulate"], s["ws"])
    return s["grads"]


def _own_norm_fwd(s, c):
    s["mtx"].mtx_block_norm_forward(s["desc"], s["h"], s["x"], s["h_out"], s["y"], s["stats"])
    return {"h": s["h_out"], "y": s["y"]}


def _slots(s, c):
    """The parameters' gradients in the shards' rows: name -> columns."""
    D = c["D"]
    names = [k for k in ("post_w", "post_b", "gate", "pre_w", "pre_b")
             if s[k] is not None and not (k == "gate" and c["group"])]
    return {k: s["grads"][:, i * D:(i + 1) * D] for i, k in enumerate(names)}


def _own_norm_bwd(s, c):
    d = _slots(s, c)
    s["mtx"].mtx_block_norm_backward(
        s["desc"], c["R"], s["h"], s["x"], s["stats"], s["dy"], s["dh_out"], s["dh"], s["dx"],
        d.get("post_w"), d.get("post_b"), s["dgate"] if c["group"] else d.get("gate"),
        d.get("pre_w"), d.get("pre_b"), s["ld"], s["ws"])
    out = {"dh": s["dh"], "dx": s["dx"]} | {"d_" + k: v for k, v in d.items()}
    return out | ({"d_gate": s["dgate"]} if c["gate"] and c["group"] else {})


def _own_clip_list(s, c):
    s["mtx"].mtx_clip_grads(s["clip"].handle, s["max_norm"], s["norm"])
    return {"grads": s["dst"], "norm": s["norm"]}


def _own_clip_avg(s, c):
    s["mtx"].mtx_average_clip(s["grads"], c["R"], c["n"], c["ld"], s["max_norm"], s["avg"],
                              s["norm"], s["ws"])
    return {"grads": s["avg"], "norm": s["norm"]}


_run_own = {"embed_fwd": _own_embed_fwd, "embed_bwd": _own_embed_bwd, "norm_fwd": _own_norm_fwd,
            "norm_bwd": _own_norm_bwd, "clip_list": _own_clip_list, "clip_avg": _own_clip_avg}


# ---- plain forms --------------------------------------------------------------------------------

def _plain_embed_fwd(s, c):
    t = s["tokens"].long()
    y = s["w"][t].float() * c["scale"]
    if c["pad"] >= 0:
        y = y * (t != c["pad"])[:, None]
    return y.to(TYPES[c["dtype"]])


def _plain_embed_bwd(s, c):
    R, n, V, D = c["R"], c["n"], c["V"], c["D"]
    t = s["tokens"].long()
    dy = s["dy"].float() * c["scale"]
    if c["pad"] >= 0:
        dy = dy * (t != c["pad"])[:, None]
    row = t + torch.arange(R, device="cuda").repeat_interleave(n) * V
    g = s["grads"].view(R * V, D)
    if not c["accumulate"]:
        g.zero_()
    g.index_add_(0, row, dy)
    return s["grads"]


def _plain_hat(t, layer):
    mean = t.mean(1, keepdim=True) if layer else 0.0
    r = ((t - mean).square().mean(1, keepdim=True) + EPS).rsqrt()
    return (t - mean) * r, r


def _plain_gate(s, c):
    if s["gate"] is None:
        return 1.0
    return s["gate"].repeat_interleave(c["group"] or c["rows"], 0)


def _plain_norm_fwd(s, c):
    dt = TYPES[c["dtype"]]
    u = s["x"].float()
    if c["post"]:
        u = _plain_hat(u, c["layer"])[0] * s["post_w"]
        u = u + s["post_b"] if c["layer"] else u
    h = s["h"].float() + c["scale"] * _plain_gate(s, c) * u
    y = _plain_hat(h, c["layer"])[0] * s["pre_w"]
    y = y + s["pre_b"] if c["layer"] else y
    return {"h": h.to(dt), "y": y.to(dt)}


def _plain_pull(g, hat, r, layer):
    """Gradient through (t - mean) r with respect to t."""
    g = g - hat * (g * hat).mean(1, keepdim=True) - (g.mean(1, keepdim=True) if layer else 0.0)
    return g * r


def _plain_norm_bwd(s, c):
    dt, R, D, N = TYPES[c["dtype"]], c["R"], c["D"], c["rows"]
    st, layer = s["stats"], c["layer"]

    def shard(t):
        return t.view(R, N // R, D).sum(1)

    dy = s["dy"].float()
    hat = (s["h"].float() - st[:, 2:3]) * st[:, 3:4]
    d = {"d_pre_w": shard(dy * hat)}
    if layer:
        d["d_pre_b"] = shard(dy)
    dh = s["dh_out"].float() + _plain_pull(dy * s["pre_w"], hat, st[:, 3:4], layer)
    x = s["x"].float()
    du = c["scale"] * _plain_gate(s, c) * dh
    u, dx = x, du
    if c["post"]:
        xhat = (x - st[:, 0:1]) * st[:, 1:2]
        u = xhat * s["post_w"]
        d["d_post_w"] = shard(du * xhat)
        if layer:
            u = u + s["post_b"]
            d["d_post_b"] = shard(du)
        dx = _plain_pull(du * s["post_w"], xhat, st[:, 1:2], layer)
    if c["gate"]:
        e = c["scale"] * dh * u
        d["d_gate"] = e.view(-1, c["group"], D).sum(1) if c["group"] else shard(e)
    return {"dh": dh.to(dt), "dx": dx.to(dt)} | d


def _plain_scale(g, total, max_norm):
    norm = total.sqrt()
    coef = torch.where(norm > max_norm, max_norm / norm, torch.ones_like(norm))
    return {"grads": g * coef.float(), "norm": norm.float().view(1)}


def _plain_clip_list(s, c):
    flat = torch.cat([t.view(-1) for t in s["src"]]).float()
    return _plain_scale(flat, flat.square().sum().double(), s["max_norm"])


def _plain_clip_avg(s, c):
    g = s["grads"][:, :c["n"]].sum(0) / c["R"]
    return _plain_scale(g, g.square().sum().double(), s["max_norm"])


_run_plain = {"embed_fwd": _plain_embed_fwd, "embed_bwd": _plain_embed_bwd,
              "norm_fwd": _plain_norm_fwd, "norm_bwd": _plain_norm_bwd,
              "clip_list": _plain_clip_list, "clip_avg": _plain_clip_avg}


# ---- what a pass cannot do without ------------------------------------------------------------

def work(case):
    c, op = case, case["op"]
    size = {"f32": 4, "bf16": 2}
    if op == "embed_fwd":
        N = c["R"] * c["n"]
        return {"bytes": N * (4 + c["D"] * (size[c["table"]] + size[c["dtype"]])),
                "flops": N * c["D"]}
    if op == "embed_bwd":
        N, D, V, R = c["R"] * c["n"], c["D"], c["V"], c["R"]
        # distinct tokens expected of n draws with p(rank) ~ 1 / rank
        hit = sum(-math.expm1(c["n"] * math.log1p(-min(0.999, math.log1p(1 / k) / math.log(V))))
                  * max(1, k // 64) for k in _ranks(V))
        table = 2 * R * min(hit, c["n"], V) if c["accumulate"] else R * V
        return {"bytes": int(4 * N + N * (1 - c["padded"]) * D * size[c["dtype"]] + table * D * 4),
                "flops": 2 * N * D}
    if op == "norm_fwd":
        e, N, D = size[c["dtype"]], c["rows"], c["D"]
        gates = (N // c["group"] if c["group"] else 1) * c["gate"]
        return {"bytes": N * D * e * 4 + 16 * N + 4 * D * (2 + gates),
                "flops": N * D * (16 if c["post"] else 9)}
    if op == "norm_bwd":
        e, N, D = size[c["dtype"]], c["rows"], c["D"]
        gates = (N // c["group"] if c["group"] else c["R"]) * c["gate"]
        return {"bytes": N * D * e * 6 + 16 * N + 4 * D * (2 * c["R"] + 2 * gates),
                "flops": N * D * (30 if c["post"] else 16)}
    if op == "clip_list":
        n = sum(_sizes(c, 11))
        return {"bytes": n * (size[c["dtype"]] + 4), "flops": 3 * n}
    return {"bytes": 4 * c["n"] * (c["R"] + 1), "flops": c["n"] * (c["R"] + 3)}


def _ranks(V):
    """Ranks 1 .. V, thinned: each k stands for max(1, k // 64) ranks."""
    k = 1
    while k <= V:
        yield k
        k += max(1, k // 64)


# ---- the definitions in 64 bits -----------------------------------------------------------------

def exact(case, seed):
    c, op = case, case["op"]
    s = prepare(case, seed)
    if op == "embed_fwd":
        table = torch.cat([s["w"].double() * c["scale"],
                           torch.zeros(1, c["D"], device="cuda", dtype=torch.float64)])
        t = s["tokens"].long()
        return table.index_select(0, torch.where(t == c["pad"], c["V"], t))
    if op == "embed_bwd":
        R, n, V, D = c["R"], c["n"], c["V"], c["D"]
        t = s["tokens"].long().view(R, n)
        dy = s["dy"].double().view(R, n, D)
        out = s["grads"].double().view(R, V, D) if c["accumulate"] else torch.zeros(
            R, V, D, device="cuda", dtype=torch.float64)
        for r in range(R):
            kept = t[r] != c["pad"]
            order = t[r][kept].argsort(stable=True)
            tok, count = t[r][kept][order].unique_consecutive(return_counts=True)
            ends = count.cumsum(0)
            sums = torch.cat([torch.zeros(1, D, device="cuda", dtype=torch.float64),
                              dy[r][kept][order].cumsum(0)])
            out[r, tok] += c["scale"] * (sums[ends] - sums[ends - count])
        return out.view(R, V * D)
    if op.startswith("norm"):
        return _exact_norm(c, s)
    if op == "clip_list":
        g = torch.cat([t.double() for t in s["src"]])
    else:
        g = s["grads"][:, :c["n"]].double().mean(0)
    norm = torch.dot(g, g).sqrt()
    return {"grads": g * (s["max_norm"] / norm).clamp(max=1.0), "norm": norm.view(1)}


def _exact_norm(c, s):
    """The forward formula in 64 bits; the backward pass by differentiating it."""
    N, D, R = c["rows"], c["D"], c["R"]
    back = c["op"] == "norm_bwd"
    leaf = {}
    for k in ("post_w", "post_b", "pre_w", "pre_b"):
        if s[k] is not None:
            leaf[k] = s[k].double().expand(R, D).contiguous().requires_grad_(back)
    if c["gate"]:
        G = N // c["group"] if c["group"] else R
        leaf["gate"] = s["gate"].double().expand(G, D).contiguous().requires_grad_(back)

    def rows(p):
        return p.repeat_interleave(N // p.shape[0], 0)

    def normed(t, w, b):
        if c["layer"]:
            t = t - t.mean(-1, keepdim=True)
        t = t / torch.sqrt((t * t).mean(-1, keepdim=True) + EPS) * rows(leaf[w])
        return t + rows(leaf[b]) if b in leaf else t

    x = s["x"].double().requires_grad_(back)
    step = normed(x, "post_w", "post_b") if c["post"] else x
    step = c["scale"] * step * rows(leaf["gate"]) if c["gate"] else c["scale"] * step
    if not back:
        h = s["h"].double() + step
        return {"h": h, "y": normed(h, "pre_w", "pre_b")}
    # s["h"] holds the stream after the addition
    h = s["h"].double().requires_grad_(True)
    y = normed(h, "pre_w", "pre_b")
    first = {k: leaf[k] for k in ("pre_w", "pre_b") if k in leaf}
    got = torch.autograd.grad(y, [h, *first.values()], s["dy"].double())
    dh = s["dh_out"].double() + got[0]
    out = {"dh": dh} | {"d_" + k: v for k, v in zip(first, got[1:])}
    rest = {k: v for k, v in leaf.items() if k not in first}
    got = torch.autograd.grad(step, [x, *rest.values()], dh)
    return out | {"dx": got[0]} | {"d_" + k: v for k, v in zip(rest, got[1:])}
