"""Performance cases of the operators that complete a Mixture-of-Experts layer on
one GPU: the experts' networks on the dispatched rows and their gradients, the
whole layer for a few tokens, and the clipping of the gradients by their global
norm.

A case is a dict of plain values; `op` names the operator that one pass runs:

  experts      the expert networks act(xe w1 + b1) w2 + b2 on the [E, C, d] rows
               that a dispatch left, counts[e] of them in use; with `keep` the
               pre-activations are returned for the backward pass
  experts_bwd  their gradients: of the rows, both weights and both biases
  layer        gate, experts and combine of a batch of few tokens, no capacity
  clip         the global norm of many gradients, and the gradients scaled to it

`run` computes them in elementary torch operations, or, where `own` is true, by
the library's calls.  Inputs are normal draws as a normalised layer has them,
weights scaled by one over the root of their input width.
"""

import math

import torch

own = False

_DEV = "cuda"


# ---------------------------------------------------------------- cases

def _experts(op, dtype, E, C, d, h, act, gated, fill=1.0, keep=False, name=None):
    """fill: mean share of the C slots in use; counts are drawn around it and capped at C."""
    c = dict(op=op, dtype=dtype, E=E, C=C, d=d, h=h, act=act, gated=gated, fill=fill, keep=keep)
    return c if name is None else dict(c, name=name)


def _layer(dtype, S, d, E, k, h, act, gated, kind="topk", normalize=1, name=None):
    c = dict(op="layer", dtype=dtype, S=S, d=d, E=E, k=k, h=h, act=act, gated=gated, kind=kind, normalize=normalize)
    return c if name is None else dict(c, name=name)


def _clip(dtype, layers, d, E, h, scale, name=None):
    """The gradients of `layers` layers; scale: their norm over the allowed one."""
    c = dict(op="clip", dtype=dtype, layers=layers, d=d, E=E, h=h, scale=scale)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # the small Switch layer in fp32: 1024 tokens, width 256, 8 experts
        _experts("experts", "f32", 8, 128, 256, 1024, "relu", False, fill=0.9, keep=True, name="experts_switch_f32"),
        # a ragged inference batch whose sizes are no powers of two, half of the slots unused
        _experts("experts", "bf16", 60, 313, 1400, 1000, "silu", True, fill=0.5, name="experts_odd_bf16"),
        # the GShard layer in training: top-2 of 16 experts, 8192 tokens, capacity factor 1.25
        _experts("experts", "bf16", 16, 1280, 1024, 4096, "gelu", False, fill=0.8, keep=True,
                 name="experts_gshard_bf16"),
        # expert prototyping at the full batch: 32768 tokens with four choices each, gated experts
        _experts("experts", "bf16", 64, 2560, 2048, 2048, "silu", True, fill=0.8, keep=True,
                 name="experts_ktop1_bf16"),
        # gradients of the small fp32 layer, of the GShard layer, and of 64 wide experts
        # (32768 tokens, capacity factor 1), where the weights' gradients are the most of it
        _experts("experts_bwd", "f32", 8, 128, 256, 1024, "relu", False, fill=0.9, name="bwd_switch_f32"),
        _experts("experts_bwd", "bf16", 16, 1280, 1024, 4096, "silu", True, fill=0.8, name="bwd_gshard_bf16"),
        _experts("experts_bwd", "bf16", 64, 512, 2048, 8192, "gelu", False, fill=0.9, name="bwd_wide_bf16"),
        # one token of one request: the weights of its two experts are all there is to read
        _layer("bf16", 1, 2048, 64, 2, 8192, "gelu", False, name="layer_one_bf16"),
        # one decode step of 32 requests on gated experts: most experts get a token
        _layer("bf16", 32, 2048, 64, 2, 2048, "silu", True, name="layer_decode_bf16"),
        # a larger step in fp32, four groups of experts, one of each
        _layer("f32", 100, 1024, 16, 4, 4096, "relu", False, kind="ktop1", normalize=0, name="layer_batch_f32"),
        # the gradients of one small layer: launches are what it takes
        _clip("f32", 1, 256, 8, 1024, 4.0, name="clip_switch_f32"),
        # the gradients of six GShard layers, 0.8 billion values in 36 tensors
        _clip("bf16", 6, 1024, 16, 4096, 4.0, name="clip_gshard_bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A row length: whole 16-byte pieces in both types; half of them multiples of 64."""
    n = _log(rng, lo, hi)
    return max(64, n // 64 * 64) if rng.random() < 0.5 else max(8, n // 8 * 8)


def draw(rng):
    op = rng.choice(["experts", "experts", "experts_bwd", "experts_bwd", "layer", "layer", "clip"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    act = rng.choice(["relu", "gelu", "silu", "silu"])
    gated = rng.random() < 0.5
    if op == "clip":
        d, h, E, layers = _width(rng, 128, 2048), _width(rng, 256, 8192), _log(rng, 4, 64), rng.randint(1, 6)
        layers = max(1, min(layers, int(4e8 // (2.0 * E * d * h))))
        while 2 * E * d * h > 4e8:
            E //= 2
        return _clip(dtype, layers, d, E, h, rng.choice([0.5, 4.0, 100.0]))
    d, h = _width(rng, 64, 4096), _width(rng, 64, 8192)
    if op == "layer":
        E, k, kind = _log(rng, 4, 128), rng.choice([1, 2, 2, 3, 4, 8]), rng.choice(["topk", "topk", "ktop1"])
        E = max(k, E // k * k)
        while E * d * h > 2 ** 30:
            E -= k
            if E < k:
                E, h = k, h // 2 // 8 * 8
        return _layer(dtype, _log(rng, 1, 256), d, E, k, h, act, gated, kind=kind,
                      normalize=rng.randint(0, 1) if kind == "topk" else 0)
    E = _log(rng, 2, 128)
    C = _log(rng, 1, 4096)
    # no more work than the largest listed case of its type
    most = (2.0 ** 37 if dtype == "f32" else 2.0 ** 39) / (3 if op == "experts_bwd" else 1)
    while E * d * h > 2 ** 29:
        E = max(1, E // 2)
        h = h if E > 1 else max(64, h // 2)
    while E * C * float(d) * h > most or E * C * (2 * h + d) > 2 ** 29:
        C = max(1, C // 2 + C % 2)
    return _experts(op, dtype, E, C, d, h, act, gated, fill=rng.choice([0.3, 0.8, 1.0, 2.0]),
                    keep=op == "experts" and rng.random() < 0.5)


# ---------------------------------------------------------------- inputs

def _dt(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def prepare(case, seed):
    c = case
    g = torch.Generator(device=_DEV)
    g.manual_seed(seed)
    dt = _dt(c)

    def normal(*shape, dtype=dt, scale=1.0):
        return torch.randn(shape, generator=g, device=_DEV, dtype=dtype).mul_(scale)

    d, h, E = c["d"], c["h"], c["E"]
    if c["op"] == "clip":
        grads = []
        for _ in range(c["layers"]):
            grads += [normal(E, d, h, scale=1e-3), normal(E, h, dtype=torch.float32, scale=1e-3),
                      normal(E, h, d, scale=1e-3), normal(E, d, dtype=torch.float32, scale=1e-3),
                      normal(d, E, dtype=torch.float32, scale=1e-2), normal(E, dtype=torch.float32, scale=1e-2)]
        values = float(c["layers"]) * (2.0 * E * d * h + E * h + E * d + 100.0 * (d * E + E))
        return dict(c=c, grads=grads, out=[torch.empty_like(t) for t in grads],
                    max_norm=1e-3 * math.sqrt(values) / c["scale"])
    h1 = 2 * h if c["gated"] else h
    s = dict(c=c, w1=normal(E, d, h1, scale=d ** -0.5), w2=normal(E, h, d, scale=h ** -0.5),
             b1=normal(E, h1, dtype=torch.float32, scale=0.1), b2=normal(E, d, dtype=torch.float32, scale=0.1))
    if c["op"] == "layer":
        s["x"] = normal(c["S"], d)
        s["wg"] = normal(d, E, scale=d ** -0.5)
        s["bg"] = normal(E, dtype=torch.float32, scale=0.1)
        return s
    C = c["C"]
    # rows in use per expert: a skewed load cut at the capacity, an idle expert now and then
    load = torch.ceil(torch.rand((E,), generator=g, device=_DEV) * 2.0 * c["fill"] * C).clamp(1.0, float(C))
    idle = torch.rand((E,), generator=g, device=_DEV) < 0.03
    idle[0] = False
    s["counts"] = torch.where(idle, torch.zeros_like(load), load).to(torch.int32)
    used = torch.arange(C, device=_DEV)[None, :, None] < s["counts"][:, None, None]
    s["used"] = used
    s["xe"] = normal(E, C, d) * used  # a dispatch leaves zero rows in empty slots
    if c["op"] == "experts_bwd":
        # what the forward pass kept, and the rows that the combine's gradient left
        pre, hidden = _hidden(c, s["xe"].float(), s["w1"].float(), s["b1"])
        s["pre"], s["hidden"] = (pre * used).to(dt), (hidden * used).to(dt)
        s["dye"] = normal(E, C, d) * used
    return s


# ---------------------------------------------------------------- the plain forms, in fp32

_GELU0, _GELU1 = 0.7978845608028654, 0.044715


def _act(name, a):
    if name == "relu":
        return a.clamp(min=0.0)
    if name == "silu":
        return a / (1.0 + torch.exp(-a))
    # the tanh form: a * sigmoid(2 u)
    return a / (1.0 + torch.exp(-2.0 * _GELU0 * (a + _GELU1 * a * a * a)))


def _act_grad(name, a):
    if name == "relu":
        return (a > 0.0).to(a.dtype)
    if name == "silu":
        p = 1.0 / (1.0 + torch.exp(-a))
        return p * (1.0 + a * (1.0 - p))
    p = 1.0 / (1.0 + torch.exp(-2.0 * _GELU0 * (a + _GELU1 * a * a * a)))
    return p + a * p * (1.0 - p) * 2.0 * _GELU0 * (1.0 + 3.0 * _GELU1 * a * a)


def _hidden(c, x, w1, b1):
    pre = torch.matmul(x, w1) + b1[:, None, :]
    if c["gated"]:
        return pre, _act(c["act"], pre[..., : c["h"]]) * pre[..., c["h"]:]
    return pre, _act(c["act"], pre)


def _plain_experts(c, s):
    dt, used = _dt(c), s["used"]
    x = torch.where(used, s["xe"], 0).float()
    pre, hidden = _hidden(c, x, s["w1"].float(), s["b1"])
    ye = torch.matmul(hidden, s["w2"].float()) + s["b2"][:, None, :]
    out = {"ye": (ye * used).to(dt)}
    if c["keep"]:
        out["pre"], out["hidden"] = (pre * used).to(dt), (hidden * used).to(dt)
    return out


def _plain_experts_bwd(c, s):
    dt, used, h = _dt(c), s["used"], c["h"]
    dy = torch.where(used, s["dye"], 0).float()
    x = torch.where(used, s["xe"], 0).float()
    pre = torch.where(used, s["pre"], 0).float()
    hidden = torch.where(used, s["hidden"], 0).float()
    dh = torch.matmul(dy, s["w2"].float().transpose(1, 2))
    if c["gated"]:
        a, u = pre[..., :h], pre[..., h:]
        dpre = torch.cat([dh * u * _act_grad(c["act"], a), dh * _act(c["act"], a)], dim=2)
    else:
        dpre = dh * _act_grad(c["act"], pre)
    return {"dxe": torch.matmul(dpre, s["w1"].float().transpose(1, 2)).to(dt),
            "dw1": torch.matmul(x.transpose(1, 2), dpre).to(dt), "db1": dpre.sum(dim=1),
            "dw2": torch.matmul(hidden.transpose(1, 2), dy).to(dt), "db2": dy.sum(dim=1)}


def _plain_layer(c, s):
    S, E, k = c["S"], c["E"], c["k"]
    x = s["x"].float()
    # 64 bits: the choice between near logits
    logits = torch.matmul(s["x"].double(), s["wg"].double()) + s["bg"].double()
    if c["kind"] == "ktop1":
        lg = logits.view(S, k, E // k)
        best, at = torch.sort(lg, dim=2, descending=True, stable=True)
        weights = 1.0 / torch.exp(lg - best[..., :1]).sum(dim=2)
        ids = at[..., 0] + torch.arange(k, device=x.device)[None, :] * (E // k)
    else:
        best, at = torch.sort(logits, dim=1, descending=True, stable=True)
        ids, e = at[:, :k], torch.exp(best - best[:, :1])
        weights = e[:, :k] / (e[:, :k] if c["normalize"] else e).sum(dim=1, keepdim=True)
    weights = weights.float()
    if S * k <= E:
        # the chosen experts' weights alone, one copy for each choice
        f = ids.reshape(-1)
        xr = x.repeat_interleave(k, dim=0)[:, None, :]
        _, hidden = _hidden(c, xr, s["w1"][f].float(), s["b1"][f])
        ye = torch.matmul(hidden, s["w2"][f].float())[:, 0, :] + s["b2"][f]
        y = (ye.view(S, k, -1) * weights[:, :, None]).sum(dim=1)
    else:
        # every expert on every token, weighted by the choices
        share = torch.zeros((S, E), device=x.device).scatter_(1, ids, weights)
        _, hidden = _hidden(c, x[None], s["w1"].float(), s["b1"])
        ye = torch.matmul(hidden, s["w2"].float()) + s["b2"][:, None, :]
        y = (ye * share.t()[:, :, None]).sum(dim=0)
    return {"y": y.to(_dt(c)), "ids": ids.to(torch.int32), "weights": weights}


def _plain_clip(s):
    total = torch.stack([t.double().square().sum() for t in s["grads"]]).sum()
    norm = torch.sqrt(total)
    scale = torch.clamp(s["max_norm"] / norm, max=1.0).float()
    return {"norm": norm.float().reshape(1),
            "grads": [o.copy_(t.float() * scale) for t, o in zip(s["grads"], s["out"])]}


def run(state):
    s, c = state, state["c"]
    if own:
        import paper_2203_14685_amd as hm
        if c["op"] == "clip":
            norm = hm.clip_grads(s["grads"], s["max_norm"], out=s["out"])
            return {"norm": norm, "grads": s["out"]}
        act = {"relu": hm.MOE_ACT_RELU, "gelu": hm.MOE_ACT_GELU, "silu": hm.MOE_ACT_SILU}[c["act"]]
        if c["op"] == "experts":
            o = hm.experts(s["xe"], s["w1"], s["w2"], b1=s["b1"], b2=s["b2"], counts=s["counts"], act=act,
                           gated=c["gated"], want_pre=c["keep"])
            return {key: o[key] for key in (("ye", "pre", "hidden") if c["keep"] else ("ye",))}
        if c["op"] == "experts_bwd":
            return hm.experts_bwd(s["dye"], s["xe"], s["w1"], s["w2"], s["pre"], s["hidden"], counts=s["counts"],
                                  act=act, gated=c["gated"])
        kind = hm.MOE_GATE_KTOP1 if c["kind"] == "ktop1" else hm.MOE_GATE_TOPK
        return hm.token_layer(s["x"], s["w1"], s["w2"], b1=s["b1"], b2=s["b2"], act=act, gated=c["gated"], kind=kind,
                              k=c["k"], wg=s["wg"], bias=s["bg"], normalize=c["normalize"])
    if c["op"] == "clip":
        return _plain_clip(s)
    return {"experts": _plain_experts, "experts_bwd": _plain_experts_bwd, "layer": _plain_layer}[c["op"]](c, s)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    c = case
    d, h, E = c["d"], c["h"], c["E"]
    b = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "clip":
        big, small = c["layers"] * 2 * E * d * h, c["layers"] * (E * h + 2 * E * d + E)
        return {"bytes": 2 * (b * big + 4 * small) + 4, "flops": 3 * (big + small)}
    h1 = 2 * h if c["gated"] else h
    weights = E * (d * h1 + h * d)
    if c["op"] == "layer":
        S, k = c["S"], c["k"]
        # experts that at least one of S * k even choices takes
        hit = E * (1.0 - (1.0 - 1.0 / E) ** (S * k)) if S > 1 else k
        return {"bytes": int(b * (hit / E * weights + 2 * S * d + d * E) + 4 * (hit * (h1 + d) + E) + 8 * S * k),
                "flops": int(2 * S * d * E + 2 * S * k * (d * h1 + h * d))}
    # rows in use: the mean of a uniform load on [0, 2 fill C] cut at C, 3 % of the experts idle
    C, f = c["C"], c["fill"]
    rows = 0.97 * E * C * (f if f <= 0.5 else 1.0 - 0.25 / f)
    if c["op"] == "experts":
        out = E * C * (d + (h1 + h if c["keep"] else 0))
        return {"bytes": int(b * (weights + rows * d + out) + 4 * E * (h1 + d + 1)),
                "flops": int(2 * rows * (d * h1 + h * d))}
    return {"bytes": int(b * (2 * weights + rows * (2 * d + h1 + h) + E * C * d) + 4 * E * (h1 + d + 1)),
            "flops": int(4 * rows * (d * h1 + h * d))}


# ---------------------------------------------------------------- from the definitions, in 64 bits

def _act64(name, a):
    """The activation and its derivative."""
    if name == "relu":
        return torch.where(a > 0, a, torch.zeros_like(a)), torch.where(a > 0, 1.0, 0.0).double()
    if name == "silu":
        p = torch.sigmoid(a)
        return a * p, p + a * p * torch.sigmoid(-a)
    u = math.sqrt(2.0 / math.pi) * (a + 0.044715 * a ** 3)
    t = torch.tanh(u)
    return 0.5 * a * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * a * (1.0 - t * t) * math.sqrt(2.0 / math.pi) * (1.0 + 3 * 0.044715 * a * a)


def _net64(c, x, w1, b1, w2, b2):
    pre = x @ w1 + b1
    if c["gated"]:
        hidden = _act64(c["act"], pre[:, : c["h"]])[0] * pre[:, c["h"]:]
    else:
        hidden = _act64(c["act"], pre)[0]
    return pre, hidden, hidden @ w2 + b2


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    f64 = dict(dtype=torch.float64, device=_DEV)
    if c["op"] == "clip":
        total = sum(float((t.double() ** 2).sum()) for t in s["grads"])
        norm = math.sqrt(total)
        scale = min(1.0, s["max_norm"] / norm)
        return {"norm": torch.full((1,), norm, **f64), "grads": [t.double() * scale for t in s["grads"]]}
    d, h, E = c["d"], c["h"], c["E"]
    h1 = 2 * h if c["gated"] else h
    if c["op"] == "layer":
        S, k = c["S"], c["k"]
        logits = s["x"].double() @ s["wg"].double() + s["bg"].double()
        host = logits.tolist()
        ids = torch.empty((S, k), dtype=torch.int64)
        weights = torch.empty((S, k), dtype=torch.float64)
        for t in range(S):
            row = host[t]
            if c["kind"] == "ktop1":
                G = E // k
                chosen = [max(range(r * G, r * G + G), key=lambda e: (row[e], -e)) for r in range(k)]
                total = [sum(math.exp(v - row[chosen[r]]) for v in row[r * G: r * G + G]) for r in range(k)]
            else:
                chosen = sorted(range(E), key=lambda e: (-row[e], e))[:k]
                over = [row[e] for e in chosen] if c["normalize"] else row
                total = [sum(math.exp(v - row[e]) for v in over) for e in chosen]
            ids[t] = torch.tensor(chosen)
            weights[t] = torch.tensor([1.0 / z for z in total], dtype=torch.float64)
        ids, weights = ids.to(_DEV), weights.to(_DEV)
        y = torch.zeros((S, d), **f64)
        for e in range(E):
            t, r = torch.nonzero(ids == e, as_tuple=True)
            if t.numel():
                ye = _net64(c, s["x"][t].double(), s["w1"][e].double(), s["b1"][e].double(), s["w2"][e].double(),
                            s["b2"][e].double())[2]
                y.index_add_(0, t, ye * weights[t, r][:, None])
        return {"y": y, "ids": None, "weights": weights}
    C, counts = c["C"], s["counts"].tolist()
    if c["op"] == "experts":
        out = {"ye": torch.zeros((E, C, d), **f64)}
        if c["keep"]:
            out.update(pre=torch.zeros((E, C, h1), **f64), hidden=torch.zeros((E, C, h), **f64))
        for e, n in enumerate(counts):
            pre, hidden, ye = _net64(c, s["xe"][e, :n].double(), s["w1"][e].double(), s["b1"][e].double(),
                                     s["w2"][e].double(), s["b2"][e].double())
            out["ye"][e, :n] = ye
            if c["keep"]:
                out["pre"][e, :n], out["hidden"][e, :n] = pre, hidden
        return out
    out = {"dxe": torch.zeros((E, C, d), **f64), "dw1": torch.zeros((E, d, h1), **f64),
           "db1": torch.zeros((E, h1), **f64), "dw2": torch.zeros((E, h, d), **f64), "db2": torch.zeros((E, d), **f64)}
    for e, n in enumerate(counts):
        x, dy = s["xe"][e, :n].double(), s["dye"][e, :n].double()
        pre, hidden = s["pre"][e, :n].double(), s["hidden"][e, :n].double()
        dh = dy @ s["w2"][e].double().t()
        if c["gated"]:
            a, da = _act64(c["act"], pre[:, :h])
            dpre = torch.cat([dh * pre[:, h:] * da, dh * a], dim=1)
        else:
            dpre = dh * _act64(c["act"], pre)[1]
        out["dxe"][e, :n] = dpre @ s["w1"][e].double().t()
        out["dw1"][e], out["db1"][e] = x.t() @ dpre, dpre.sum(dim=0)
        out["dw2"][e], out["db2"][e] = hidden.t() @ dy, dy.sum(dim=0)
    return out
