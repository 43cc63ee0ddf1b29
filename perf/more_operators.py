"""Performance cases of what surrounds a Mixture-of-Experts layer on one GPU: the
embedding rows that it starts from and their gradient, dropout on rows and inside
the experts, and the expert networks and the layer for a few tokens in 8-bit
integers.

A case is a dict of plain values; `op` names the operator that one pass runs:

  embed        scaled rows of a table by token id
  embed_bwd    the table's gradient: the rows' gradients summed per token id; with
               `accumulate` on top of a gradient that is there already
  drop         rows with elements dropped, scaled, on top of a residual if there is one
  drop_net     the expert networks with dropout of the hidden rows (training: the
               pre-activations are kept)
  drop_net_bwd their gradients
  int8_net     the expert networks with rows and weights in 8-bit integers, a scale per
               row and per column of the weights
  int8_layer   gate, 8-bit experts and weighted sum of a batch of few tokens

`run` computes them in elementary torch operations, or, where `own` is true, by
the library's calls.  Inputs are normal draws as a normalised layer has them,
weights scaled by one over the root of their input width, token ids by a power law
as text has them.
"""

import math

import torch

own = False

_DEV = "cuda"
_M32 = 0xFFFFFFFF


# ---------------------------------------------------------------- cases

def _named(case, name):
    return case if name is None else dict(case, name=name)


def _embed(dtype, T, V, d, zipf=1.1, scale=1.0, name=None):
    """zipf: exponent of the ids' power law, 0 for even ones."""
    return _named(dict(op="embed", dtype=dtype, T=T, V=V, d=d, zipf=zipf, scale=scale), name)


def _embed_bwd(dtype, T, V, d, zipf=1.1, scale=1.0, accumulate=False, name=None):
    return _named(dict(op="embed_bwd", dtype=dtype, T=T, V=V, d=d, zipf=zipf, scale=scale, accumulate=accumulate), name)


def _drop(dtype, S, d, p, residual, name=None):
    return _named(dict(op="drop", dtype=dtype, S=S, d=d, p=p, residual=residual), name)


def _net(op, dtype, E, C, d, h, act, gated, fill=1.0, p=0.0, name=None):
    """fill: mean share of the C slots in use; counts are drawn around it and capped at C."""
    return _named(dict(op=op, dtype=dtype, E=E, C=C, d=d, h=h, act=act, gated=gated, fill=fill, p=p), name)


def _layer(S, d, E, k, h, act, gated, kind="topk", normalize=1, name=None):
    return _named(dict(op="int8_layer", dtype="bf16", S=S, d=d, E=E, k=k, h=h, act=act, gated=gated, kind=kind,
                       normalize=normalize), name)


def listed():
    return [
        # the rows of one decode step of 32 requests: latency
        _embed("bf16", 32, 50257, 2048, name="embed_decode_bf16"),
        # the full batch of the hash-routed layer, 65536 tokens of width 4096
        _embed("bf16", 65536, 50257, 4096, scale=64.0, name="embed_hash_bf16"),
        # the table's gradient of the small Switch layer's 1024 tokens: most of it is zero rows
        _embed_bwd("f32", 1024, 50257, 256, name="embed_bwd_switch_f32"),
        # of the hash-routed batch: the most frequent token stands for a tenth of the rows
        _embed_bwd("bf16", 65536, 50257, 4096, scale=64.0, name="embed_bwd_hash_bf16"),
        # dropout on the small layer's output before the residual sum: latency
        _drop("f32", 1024, 256, 0.1, True, name="drop_switch_f32"),
        # and at the batch of the prototyping layer, 32768 tokens of width 2048
        _drop("bf16", 32768, 2048, 0.1, True, name="drop_ktop1_bf16"),
        # the GShard layer in training with expert dropout: top-2 of 16 experts, 8192 tokens
        _net("drop_net", "bf16", 16, 1280, 1024, 4096, "gelu", False, fill=0.8, p=0.4, name="drop_net_gshard_bf16"),
        # the gradients of the small Switch layer with expert dropout
        _net("drop_net_bwd", "f32", 8, 128, 256, 1024, "relu", False, fill=0.9, p=0.4, name="drop_net_bwd_switch_f32"),
        # a ragged inference batch in 8 bits whose sizes are no powers of two, half of the slots unused
        _net("int8_net", "bf16", 60, 313, 1408, 1008, "silu", True, fill=0.5, name="int8_net_odd"),
        # expert prototyping at the full batch, gated experts: 32768 tokens with four choices each
        _net("int8_net", "bf16", 64, 2560, 2048, 2048, "silu", True, fill=0.8, name="int8_net_ktop1"),
        # one token of one request: the weights of its two experts are all there is to read
        _layer(1, 2048, 64, 2, 8192, "gelu", False, name="int8_layer_one"),
        # one decode step of 32 requests on gated experts: most experts get a token
        _layer(32, 2048, 64, 2, 2048, "silu", True, name="int8_layer_decode"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi, unit):
    """A row length in whole units of 16 bytes; half of them multiples of 64."""
    n = _log(rng, lo, hi)
    return max(64, n // 64 * 64) if rng.random() < 0.5 else max(unit, n // unit * unit)


def draw(rng):
    op = rng.choice(["embed", "embed_bwd", "embed_bwd", "drop", "drop", "drop_net", "drop_net_bwd", "int8_net", "int8_net",
                     "int8_layer", "int8_layer"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op in ("embed", "embed_bwd"):
        d, V, T = _width(rng, 64, 4096, 8), _log(rng, 100, 200000), _log(rng, 1, 262144)
        zipf, scale = rng.choice([0.0, 1.1, 1.1, 1.5]), rng.choice([1.0, math.sqrt(d)])
        # no more to read and write than the largest listed case
        while (T + V) * d > (2 ** 27 if dtype == "f32" else 2 ** 28):
            T, V = (T // 2, V) if T > V else (T, V // 2)
        if op == "embed":
            return _embed(dtype, T, V, d, zipf, scale)
        return _embed_bwd(dtype, T, V, d, zipf, scale, rng.random() < 0.5)
    if op == "drop":
        S, d = _log(rng, 1, 65536), _width(rng, 64, 4096, 8)
        while S * d > 2 ** 26:
            S //= 2
        return _drop(dtype, S, d, rng.choice([0.0, 0.1, 0.3, 0.5]), rng.random() < 0.5)
    act, gated = rng.choice(["relu", "gelu", "silu", "silu"]), rng.random() < 0.5
    unit = 16 if op.startswith("int8") else 8
    d, h = _width(rng, 64, 4096, unit), _width(rng, 64, 8192, unit)
    if op == "int8_layer":
        E, k, kind = _log(rng, 4, 128), rng.choice([1, 2, 2, 3, 4, 8]), rng.choice(["topk", "topk", "ktop1"])
        E = max(k, E // k * k)
        while E * d * h > 2 ** 30:
            E -= k
            if E < k:
                E, h = k, max(16, h // 2 // 16 * 16)
        return _layer(_log(rng, 1, 256), d, E, k, h, act, gated, kind=kind,
                      normalize=rng.randint(0, 1) if kind == "topk" else 0)
    E, C = _log(rng, 2, 128), _log(rng, 1, 4096)
    # no more work than the largest listed case of its kind
    most = 2.0 ** 39 if op == "int8_net" else (2.0 ** 32 if dtype == "f32" else 2.0 ** 35.5) / (2 if op == "drop_net_bwd" else 1)
    while E * d * h > 2 ** 29:
        E = max(1, E // 2)
        h = h if E > 1 else max(64, h // 2)
    while E * C * float(d) * h > most or E * C * (2 * h + d) > 2 ** 29:
        C = max(1, C // 2 + C % 2)
    return _net(op, "bf16" if op == "int8_net" else dtype, E, C, d, h, act, gated, fill=rng.choice([0.3, 0.8, 1.0, 2.0]),
                p=0.0 if op == "int8_net" else rng.choice([0.1, 0.4]))


# ---------------------------------------------------------------- inputs

def _dt(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _draws(seed):
    g = torch.Generator(device=_DEV)
    g.manual_seed(seed)

    def normal(*shape, dtype=torch.float32, scale=1.0):
        return torch.randn(shape, generator=g, device=_DEV, dtype=dtype).mul_(scale)

    return g, normal


def _token_ids(c, g):
    """int32 ids by their power law over the ranks, in steps of the cumulative shares."""
    u = torch.rand((c["T"],), generator=g, device=_DEV, dtype=torch.float64)
    share = torch.arange(1, c["V"] + 1, device=_DEV, dtype=torch.float64) ** -c["zipf"]
    edge = torch.cumsum(share, dim=0)
    return torch.searchsorted(edge, u * edge[-1]).clamp_(max=c["V"] - 1).to(torch.int32)


def _counts(c, g):
    """Rows in use per expert: a skewed load cut at the capacity, an idle expert now and then."""
    E, C = c["E"], c["C"]
    load = torch.ceil(torch.rand((E,), generator=g, device=_DEV) * 2.0 * c["fill"] * C).clamp(1.0, float(C))
    idle = torch.rand((E,), generator=g, device=_DEV) < 0.03
    idle[0] = False
    return torch.where(idle, torch.zeros_like(load), load).to(torch.int32)


def _int8_weights(w):
    """A program's weights [E, K, N], laid out once: integers [E, N, K] and scales [E, N]."""
    w = w.transpose(1, 2).contiguous().float()
    most = w.abs().amax(dim=2)
    return torch.round(w * 127.0 / most[:, :, None]).to(torch.int8), most / 127.0


def prepare(case, seed):
    c = case
    g, normal = _draws(seed)
    dt, op = _dt(c), c["op"]
    if op in ("embed", "embed_bwd"):
        s = dict(c=c, ids=_token_ids(c, g))
        if op == "embed":
            s["table"] = normal(c["V"], c["d"], dtype=dt, scale=c["d"] ** -0.5)
        else:
            s["dy"] = normal(c["T"], c["d"], dtype=dt)
            if c["accumulate"]:
                s["there"] = normal(c["V"], c["d"], dtype=dt)
        return s
    if op == "drop":
        s = dict(c=c, seed=seed * 0x9E3779B97F4A7C15 % 2 ** 64, call=(3 << 40) + seed, x=normal(c["S"], c["d"], dtype=dt))
        s["residual"] = normal(c["S"], c["d"], dtype=dt) if c["residual"] else None
        return s
    d, h, E = c["d"], c["h"], c["E"]
    h1 = 2 * h if c["gated"] else h
    s = dict(c=c, b1=normal(E, h1, scale=0.1), b2=normal(E, d, scale=0.1))
    w1, w2 = normal(E, d, h1, dtype=dt, scale=d ** -0.5), normal(E, h, d, dtype=dt, scale=h ** -0.5)
    if op.startswith("int8"):
        s["w1"], s["s1"] = _int8_weights(w1)
        s["w2"], s["s2"] = _int8_weights(w2)
    else:
        s["w1"], s["w2"] = w1, w2
        s["seed"], s["call"] = seed * 0x9E3779B97F4A7C15 % 2 ** 64, (5 << 40) + seed
    if op == "int8_layer":
        s["x"] = normal(c["S"], d, dtype=dt)
        s["wg"] = normal(d, E, dtype=dt, scale=d ** -0.5)
        s["bg"] = normal(E, scale=0.1)
        return s
    s["counts"] = _counts(c, g)
    used = torch.arange(c["C"], device=_DEV)[None, :, None] < s["counts"][:, None, None]
    s["used"] = used
    s["xe"] = normal(E, c["C"], d, dtype=dt) * used  # a dispatch leaves zero rows in empty slots
    if op == "drop_net_bwd":
        # what the forward pass kept, and the rows that the combine's gradient left
        pre = torch.matmul(s["xe"].float(), w1.float()) + s["b1"][:, None, :]
        s["pre"] = (pre * used).to(dt)
        s["hidden"] = (_dropped(s, _hidden(c, pre)) * used).to(dt)
        s["dye"] = normal(E, c["C"], d, dtype=dt) * used
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


def _hidden(c, pre):
    if c["gated"]:
        return _act(c["act"], pre[..., : c["h"]]) * pre[..., c["h"]:]
    return _act(c["act"], pre)


def _mul32(a, m):
    """Halves of the 64-bit product of 32-bit values held in int64: (high, low)."""
    v = a * m
    return (v >> 32) & _M32, v & _M32


def _philox(n, seed, call):
    """16-bit random words of elements 0 .. n - 1: word i % 8 of block i / 8 of the Philox4x32-10
    generator (Salmon et al. 2011) with key `seed` and counter (block, call)."""
    block = torch.arange((n + 7) // 8, device=_DEV, dtype=torch.int64)
    c0, c1 = block & _M32, block >> 32
    c2, c3 = torch.full_like(block, call & _M32), torch.full_like(block, call >> 32)
    k0, k1 = seed & _M32, seed >> 32
    for _ in range(10):
        h0, l0 = _mul32(c0, 0xD2511F53)
        h1, l1 = _mul32(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & _M32, (k1 + 0xBB67AE85) & _M32
    words = torch.stack([c0 & 0xFFFF, c0 >> 16, c1 & 0xFFFF, c1 >> 16, c2 & 0xFFFF, c2 >> 16, c3 & 0xFFFF, c3 >> 16], dim=1)
    return words.reshape(-1)[:n]


def _dropped(s, v):
    """v with its elements dropped and scaled, in fp32."""
    t = round(s["c"]["p"] * 65536)
    if t == 0:
        return v
    keep = _philox(v.numel(), s["seed"], s["call"]) >= t
    return torch.where(keep.view(v.shape), v * (65536.0 / (65536 - t)), 0.0)


def _plain_embed(c, s):
    ids = s["ids"].long()
    return (s["table"][ids].float() * c["scale"]).to(_dt(c))


def _plain_embed_bwd(c, s):
    total = torch.zeros((c["V"], c["d"]), device=_DEV, dtype=torch.float32)
    total.index_add_(0, s["ids"].long(), s["dy"].float())
    total *= c["scale"]
    if not c["accumulate"]:
        return total.to(_dt(c))
    return (s["there"].float() + total).to(_dt(c))


def _plain_drop(c, s):
    y = _dropped(s, s["x"].float())
    return (y if s["residual"] is None else s["residual"].float() + y).to(_dt(c))


def _plain_drop_net(c, s):
    dt, used = _dt(c), s["used"]
    pre = torch.matmul(torch.where(used, s["xe"], 0).float(), s["w1"].float()) + s["b1"][:, None, :]
    hidden = _dropped(s, _hidden(c, pre))
    ye = torch.matmul(hidden, s["w2"].float()) + s["b2"][:, None, :]
    return {"ye": (ye * used).to(dt), "pre": (pre * used).to(dt), "hidden": (hidden * used).to(dt)}


def _plain_drop_net_bwd(c, s):
    dt, used, h = _dt(c), s["used"], c["h"]
    dy = torch.where(used, s["dye"], 0).float()
    x = torch.where(used, s["xe"], 0).float()
    pre = torch.where(used, s["pre"], 0).float()
    hidden = torch.where(used, s["hidden"], 0).float()
    dh = _dropped(s, torch.matmul(dy, s["w2"].float().transpose(1, 2)))
    if c["gated"]:
        a, u = pre[..., :h], pre[..., h:]
        dpre = torch.cat([dh * u * _act_grad(c["act"], a), dh * _act(c["act"], a)], dim=2)
    else:
        dpre = dh * _act_grad(c["act"], pre)
    return {"dxe": torch.matmul(dpre, s["w1"].float().transpose(1, 2)).to(dt),
            "dw1": torch.matmul(x.transpose(1, 2), dpre).to(dt), "db1": dpre.sum(dim=1),
            "dw2": torch.matmul(hidden.transpose(1, 2), dy).to(dt), "db2": dy.sum(dim=1)}


def _rows8(x):
    """Rows as the integers next to 127 x / max |x| (in 64 bits: half of the largest value lies on a
    border) and the scale of each."""
    most = x.abs().amax(dim=-1, keepdim=True).float()
    q = torch.round(x.double() * 127.0 / torch.where(most > 0, most, 1.0).double())
    return q.float(), most / 127.0


def _net8(c, x, w1, s1, b1, w2, s2, b2):
    """Rows x [..., n, d] through networks of integer weights [..., out, in]."""
    q, scale = _rows8(x)
    pre = torch.matmul(q, w1.float().transpose(-1, -2)) * scale * s1[..., None, :] + b1[..., None, :]
    q, scale = _rows8(_hidden(c, pre).to(_dt(c)))
    return torch.matmul(q, w2.float().transpose(-1, -2)) * scale * s2[..., None, :] + b2[..., None, :]


def _plain_int8_net(c, s):
    x = torch.where(s["used"], s["xe"], 0)
    ye = _net8(c, x, s["w1"], s["s1"], s["b1"], s["w2"], s["s2"], s["b2"])
    return {"ye": (ye * s["used"]).to(_dt(c))}


def _plain_int8_layer(c, s):
    S, E, k = c["S"], c["E"], c["k"]
    # 64 bits: the choice between near logits
    logits = torch.matmul(s["x"].double(), s["wg"].double()) + s["bg"].double()
    if c["kind"] == "ktop1":
        lg = logits.view(S, k, E // k)
        best, at = torch.sort(lg, dim=2, descending=True, stable=True)
        weights = 1.0 / torch.exp(lg - best[..., :1]).sum(dim=2)
        ids = at[..., 0] + torch.arange(k, device=_DEV)[None, :] * (E // k)
    else:
        best, at = torch.sort(logits, dim=1, descending=True, stable=True)
        ids, e = at[:, :k], torch.exp(best - best[:, :1])
        weights = e[:, :k] / (e[:, :k] if c["normalize"] else e).sum(dim=1, keepdim=True)
    weights = weights.float()
    names = ("w1", "s1", "b1", "w2", "s2", "b2")
    if S * k <= E:
        # the chosen experts' weights alone, one copy for each choice
        f = ids.reshape(-1)
        ye = _net8(c, s["x"].repeat_interleave(k, dim=0)[:, None, :], *[s[n][f] for n in names])
        y = (ye.view(S, k, -1) * weights[:, :, None]).sum(dim=1)
    else:
        # every expert on every token, weighted by the choices
        share = torch.zeros((S, E), device=_DEV).scatter_(1, ids, weights)
        ye = _net8(c, s["x"][None], *[s[n] for n in names])
        y = (ye * share.t()[:, :, None]).sum(dim=0)
    return {"y": y.to(_dt(c)), "ids": ids.to(torch.int32), "weights": weights}


def run(state):
    s, c = state, state["c"]
    op = c["op"]
    if own:
        import paper_2203_14685_amd as hm
        if op == "embed":
            return hm.embed(s["ids"], s["table"], scale=c["scale"])
        if op == "embed_bwd":
            if c["accumulate"]:
                # into a copy, so that the pass can be run again; a training step adds in place
                return hm.embed_bwd(s["dy"], s["ids"], c["V"], scale=c["scale"], dtable=s["there"].clone(), accumulate=True)
            return hm.embed_bwd(s["dy"], s["ids"], c["V"], scale=c["scale"])
        act = {"relu": hm.MOE_ACT_RELU, "gelu": hm.MOE_ACT_GELU, "silu": hm.MOE_ACT_SILU}[c["act"]] if "act" in c else None
        if op.startswith("drop"):
            mask = hm.dropout_mask(c["p"], s["seed"], s["call"])
            if op == "drop":
                return hm.dropout(s["x"], mask, residual=s["residual"])
            if op == "drop_net":
                o = hm.experts(s["xe"], s["w1"], s["w2"], b1=s["b1"], b2=s["b2"], counts=s["counts"], act=act,
                               gated=c["gated"], want_pre=True, dropout=mask)
                return {key: o[key] for key in ("ye", "pre", "hidden")}
            return hm.experts_bwd(s["dye"], s["xe"], s["w1"], s["w2"], s["pre"], s["hidden"], counts=s["counts"], act=act,
                                  gated=c["gated"], dropout=mask)
        if op == "int8_net":
            return {"ye": hm.experts_int8(s["xe"], s["w1"], s["s1"], s["w2"], s["s2"], b1=s["b1"], b2=s["b2"],
                                          counts=s["counts"], act=act, gated=c["gated"])}
        kind = hm.MOE_GATE_KTOP1 if c["kind"] == "ktop1" else hm.MOE_GATE_TOPK
        return hm.token_layer_int8(s["x"], s["w1"], s["s1"], s["w2"], s["s2"], b1=s["b1"], b2=s["b2"], act=act,
                                   gated=c["gated"], kind=kind, k=c["k"], wg=s["wg"], bias=s["bg"],
                                   normalize=c["normalize"])
    return {"embed": _plain_embed, "embed_bwd": _plain_embed_bwd, "drop": _plain_drop, "drop_net": _plain_drop_net,
            "drop_net_bwd": _plain_drop_net_bwd, "int8_net": _plain_int8_net, "int8_layer": _plain_int8_layer}[op](c, s)


# ---------------------------------------------------------------- what a pass cannot do without

def _distinct(c):
    """Expected number of different token ids among T."""
    V, T, a = c["V"], c["T"], c["zipf"]
    total = sum(r ** -a for r in range(1, V + 1))
    return sum(1.0 - math.exp(T * math.log1p(-min(1.0 - 1e-12, r ** -a / total))) for r in range(1, V + 1))


def work(case):
    c = case
    op, d = c["op"], c["d"]
    b = 2 if c["dtype"] == "bf16" else 4
    if op in ("embed", "embed_bwd"):
        T, V, rows = c["T"], c["V"], _distinct(c)
        if op == "embed":
            return {"bytes": int(b * d * (rows + T) + 4 * T), "flops": T * d}
        table = 2 * V if c["accumulate"] else V  # the pass leaves the gradient that was there as it is
        return {"bytes": int(b * d * (T + table) + 4 * T), "flops": 2 * T * d}
    if op == "drop":
        n = c["S"] * d
        return {"bytes": b * n * (3 if c["residual"] else 2), "flops": 2 * n}
    h, E = c["h"], c["E"]
    h1 = 2 * h if c["gated"] else h
    weights = E * (d * h1 + h * d)
    if op == "int8_layer":
        S, k = c["S"], c["k"]
        # experts that at least one of S * k even choices takes
        hit = E * (1.0 - (1.0 - 1.0 / E) ** (S * k)) if S > 1 else k
        return {"bytes": int(hit / E * weights + b * (2 * S * d + d * E) + 4 * (2 * hit * (h1 + d) + E) + 8 * S * k),
                "flops": int(2 * S * d * E + 2 * S * k * (d * h1 + h * d))}
    # rows in use: the mean of a uniform load on [0, 2 fill C] cut at C, 3 % of the experts idle
    C, f = c["C"], c["fill"]
    rows = 0.97 * E * C * (f if f <= 0.5 else 1.0 - 0.25 / f)
    if op == "int8_net":
        return {"bytes": int(weights + b * (rows * d + E * C * d) + 4 * E * (2 * (h1 + d) + 1)),
                "flops": int(2 * rows * (d * h1 + h * d))}
    if op == "drop_net":
        return {"bytes": int(b * (weights + rows * d + E * C * (d + h1 + h)) + 4 * E * (h1 + d + 1)),
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


def _high32(a, m):
    """The upper half of a 32-bit product, from 16-bit pieces."""
    al, ah, ml, mh = a & 0xFFFF, a >> 16, m & 0xFFFF, m >> 16
    mid = (al * ml >> 16) + (ah * ml & 0xFFFF) + (al * mh & 0xFFFF)
    return ah * mh + (ah * ml >> 16) + (al * mh >> 16) + (mid >> 16)


def _factors64(case, seed, call, n):
    """What each of n elements is multiplied by: 0, or one over the share that is kept."""
    t = round(case["p"] * 65536)
    out = torch.ones((n,), device=_DEV, dtype=torch.float64)
    if t == 0:
        return out
    step = 1 << 27
    for lo in range(0, n, step):
        i = torch.arange(lo, min(n, lo + step), device=_DEV)[::8] // 8
        x = [i & _M32, i >> 32, torch.zeros_like(i) + (call & _M32), torch.zeros_like(i) + (call >> 32)]
        key = [seed & _M32, seed >> 32]
        for r in range(10):
            a, b = x[0], x[2]
            x = [_high32(b, 0xCD9E8D57) ^ x[1] ^ key[0], (b * 0xCD9E8D57) & _M32,
                 _high32(a, 0xD2511F53) ^ x[3] ^ key[1], (a * 0xD2511F53) & _M32]
            key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
        for j in range(8):
            at = out[lo + j: lo + step: 8]
            word = (x[j // 2] >> (16 * (j % 2)))[: at.numel()] % 65536
            at.copy_(torch.where(word >= t, 65536.0 / (65536 - t), 0.0))
    return out


def _quant64(x):
    most = x.abs().max(dim=-1, keepdim=True).values
    return torch.round(127.0 * x / torch.where(most == 0, torch.ones_like(most), most)), most / 127.0


def _net64(c, x, w1, b1, w2, b2):
    """8-bit network on rows x, weights as the values that they stand for, [in, out]."""
    q, scale = _quant64(x)
    pre = (q * scale) @ w1 + b1
    hidden = _act64(c["act"], pre[:, : c["h"]])[0]
    if c["gated"]:
        hidden = hidden * pre[:, c["h"]:]
    # hidden is held in the rows' type
    q, scale = _quant64(hidden.to(_dt(c)).double())
    return (q * scale) @ w2 + b2


def _weights64(s, e):
    return [(s["w1"][e].double() * s["s1"][e].double()[:, None]).t(), s["b1"][e].double(),
            (s["w2"][e].double() * s["s2"][e].double()[:, None]).t(), s["b2"][e].double()]


def exact(case, seed):
    c = case
    op, d = c["op"], c["d"]
    s = prepare(c, seed)
    f64 = dict(dtype=torch.float64, device=_DEV)
    if op == "embed":
        return torch.index_select(s["table"], 0, s["ids"]).double() * c["scale"]
    if op == "embed_bwd":
        # sums of runs of equal ids, as differences of running sums in 64 bits, some columns at a time
        order = torch.argsort(s["ids"].long(), stable=True)
        ids = s["ids"].long()[order]
        rows, length = torch.unique_consecutive(ids, return_counts=True)
        end = torch.cumsum(length, dim=0)
        out = s["there"].double() if c["accumulate"] else torch.zeros((c["V"], d), **f64)
        for lo in range(0, d, 256):
            run_sum = torch.cumsum(s["dy"][:, lo: lo + 256].double()[order], dim=0)[end - 1]
            part = torch.diff(run_sum, dim=0, prepend=torch.zeros_like(run_sum[:1]))
            out[rows, lo: lo + 256] += part * c["scale"]
        return out
    if op == "drop":
        y = _factors64(c, s["seed"], s["call"], c["S"] * d).view(c["S"], d) * s["x"].double()
        return y if s["residual"] is None else s["residual"].double() + y
    h, E = c["h"], c["E"]
    h1 = 2 * h if c["gated"] else h
    if op == "int8_layer":
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
                y.index_add_(0, t, _net64(c, s["x"][t].double(), *_weights64(s, e)) * weights[t, r][:, None])
        return {"y": y, "ids": None, "weights": weights}
    C, counts = c["C"], s["counts"].tolist()
    if op == "int8_net":
        ye = torch.zeros((E, C, d), **f64)
        for e, n in enumerate(counts):
            if n:
                ye[e, :n] = _net64(c, s["xe"][e, :n].double(), *_weights64(s, e))
        return {"ye": ye}
    factors = _factors64(c, s["seed"], s["call"], E * C * h).view(E, C, h)
    if op == "drop_net":
        out = {key: torch.zeros((E, C, n), **f64) for key, n in (("ye", d), ("pre", h1), ("hidden", h))}
        for e, n in enumerate(counts):
            pre = s["xe"][e, :n].double() @ s["w1"][e].double() + s["b1"][e].double()
            hidden = _act64(c["act"], pre[:, :h])[0] * factors[e, :n]
            if c["gated"]:
                hidden = hidden * pre[:, h:]
            out["pre"][e, :n], out["hidden"][e, :n] = pre, hidden
            out["ye"][e, :n] = hidden @ s["w2"][e].double() + s["b2"][e].double()
        return out
    out = {"dxe": torch.zeros((E, C, d), **f64), "dw1": torch.zeros((E, d, h1), **f64),
           "db1": torch.zeros((E, h1), **f64), "dw2": torch.zeros((E, h, d), **f64), "db2": torch.zeros((E, d), **f64)}
    for e, n in enumerate(counts):
        x, dy = s["xe"][e, :n].double(), s["dye"][e, :n].double()
        pre, hidden = s["pre"][e, :n].double(), s["hidden"][e, :n].double()
        dh = dy @ s["w2"][e].double().t() * factors[e, :n]
        if c["gated"]:
            a, da = _act64(c["act"], pre[:, :h])
            dpre = torch.cat([dh * pre[:, h:] * da, dh * a], dim=1)
        else:
            dpre = dh * _act64(c["act"], pre)[1]
        out["dxe"][e, :n] = dpre @ s["w1"][e].double().t()
        out["dw1"][e], out["db1"][e] = x.t() @ dpre, dpre.sum(dim=0)
        out["dw2"][e], out["db2"][e] = hidden.t() @ dy, dy.sum(dim=0)
    return out
