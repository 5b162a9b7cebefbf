"""The way of a batch into the experts, as cases that can be measured: the norm in front of a layer, routing by scores
with a bias and groups, and the experts' products in 8 bits.

`run` is one call (or the few that belong together) on what a training or serving program holds: in elementary torch
operations where `own` is false, through the library where it is true.  Sizes are those of workloads/configs.py
(c1 .. c5) and ragged ones between them.

kinds   norm     rows to their layer norm or RMS norm, behind a residual sum where there is one; `stats`: with the
                 rows' mean and deviation, which training keeps
        dnorm    its gradients; `residual`: with the gradient that the sum gets from elsewhere
        route    scores to the chosen classes, their gates and the classes' counts; `bias`: classes are chosen by
                 score + bias, and the bias then follows the counts
        droute   the logits' gradient
        quant    rows (block 1) or weights (block 128) to 8 bits and back: every 128 values of a row, or 128 x 128 of
                 a weight, share a power of two
        product  rows of every slot times its weight, both in 8 bits
        experts  the SwiGLU experts of all slots in 8 bits, from rows in 16; `keep`: with what their backward pass reads
"""
import math

import numpy as np
import torch

own = False

EPS = float(np.float32(1e-5))
RATE = float(np.float32(1e-3))
GATE_SCALE = 2.5
BLOCK = 128               # values of a row that share a scale
TOP = 448.0               # largest e4m3 value


def _norm(kind, dtype, T, d, center=True, residual=False, stats=True):
    return {"kind": kind, "dtype": dtype, "T": T, "d": d, "center": center, "residual": residual, "stats": stats}


def _route(kind, T, E, k, score="sigmoid", bias=False, groups=1, top_groups=1, group_top=1, renorm=True):
    return {"kind": kind, "T": T, "E": E, "k": k, "score": score, "bias": bias, "groups": groups, "top_groups": top_groups,
            "group_top": group_top, "renorm": renorm}


def _quant(dtype, groups, rows, n, block):
    return {"kind": "quant", "dtype": dtype, "groups": groups, "rows": rows, "n": n, "block": block}


def _product(dtype, A, S, R, n, skew=0.2):
    return {"kind": "product", "dtype": dtype, "A": A, "S": S, "R": R, "n": n, "skew": skew}


def _experts(A, S, d, f, keep=True, skew=0.2):
    return {"kind": "experts", "dtype": "bf16", "A": A, "S": S, "d": d, "f": f, "keep": keep, "skew": skew}


def listed():
    named = [
        # serving: one step of 16 requests, the residual stream summed on the way
        ("norm of 16 tokens", _norm("norm", "bf16", 16, 4096, residual=True, stats=False)),
        # c5's batch in training: two gigabytes
        ("c5 norm", _norm("norm", "bf16", 65536, 4096, residual=True)),
        # a single-precision run of odd size
        ("ragged norm gradient f32", _norm("dnorm", "f32", 777, 1160)),
        # c5's batch, with the gradient of the residual stream
        ("c5 norm gradient", _norm("dnorm", "bf16", 65536, 4096, residual=True)),
        # serving: one step of 16 requests over c5's classes
        ("routing of 16 tokens", _route("route", 16, 128, 8, bias=True, groups=8, top_groups=4, group_top=2)),
        # c5's batch, with the step of the bias that balances the classes
        ("c5 routing", _route("route", 65536, 128, 8, bias=True, groups=8, top_groups=4, group_top=2)),
        # c4's batch in training
        ("c4 routing gradient", _route("droute", 32768, 64, 6, score="softmax")),
        # c4's dispatched rows on their way into a product
        ("c4 rows in 8 bits", _quant("bf16", 1, 196608, 2048, 1)),
        # c4's first weights after an optimizer step: every slot's
        ("c4 weights in 8 bits", _quant("bf16", 128, 2816, 2048, 128)),
        # serving: 16 tokens with two choices each over c3's experts, which streams the weights
        ("c3 product of 16 tokens", _product("bf16", 32, 8, 28672, 4096)),
        # odd sizes in every direction, single-precision results
        ("ragged product f32", _product("f32", 15009, 12, 5488, 1160, skew=0.7)),
        # c5's batch through its experts in training: 26 TFLOP
        ("c5 experts", _experts(524288, 256, 4096, 2048)),
    ]
    return [dict(c, name=name) for name, c in named]


def _log(rng, lo, hi):
    return round(math.exp(rng.uniform(math.log(lo), math.log(hi))))


def draw(rng):
    kind = rng.choice(("norm", "dnorm", "dnorm", "route", "route", "droute", "quant", "product", "product", "experts"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if kind in ("norm", "dnorm"):
        d = 8 * _log(rng, 1, 1024)
        return _norm(kind, dtype, min(_log(rng, 1, 65536), (1 << 27) // d), d, center=rng.random() < 0.5, residual=rng.random() < 0.5,
                     stats=rng.random() < 0.7)
    if kind in ("route", "droute"):
        groups = rng.choice((1, 1, 2, 4, 8))
        E = groups * _log(rng, 2, 512 // groups)
        top_groups = rng.randint(1, groups)
        k = rng.randint(1, min(16, top_groups * (E // groups)))
        return _route(kind, _log(rng, 1, 65536 if E <= 128 else 16384), E, k, score=rng.choice(("softmax", "sigmoid")), bias=rng.random() < 0.5, groups=groups,
                      top_groups=top_groups, group_top=rng.choice((1, 2)), renorm=rng.random() < 0.7)
    n, R = 8 * _log(rng, 8, 1024), 8 * _log(rng, 8, 1024)
    if kind == "quant":
        if rng.random() < 0.5:
            return _quant(dtype, 1, min(_log(rng, 1, 200000), (1 << 28) // n), n, 1)
        return _quant(dtype, min(rng.randint(1, 64), (1 << 28) // (R * n) + 1), R, n, 128)
    A, S = _log(rng, 1, 65536), _log(rng, 1, 64)
    S = min(S, (1 << 29) // (R * n) + 1)
    if kind == "product":
        return _product(dtype, min(A, (1 << 30) // R), S, R, n, skew=rng.choice((0.0, 0.5, 1.0)))
    return _experts(A, S, n, min(R, 4096), keep=rng.random() < 0.6, skew=rng.choice((0.0, 0.5, 1.0)))


# ---- sizes and work

def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _width(name):
    return 2 if name == "bf16" else 4


def _blocks(n):
    return -(-n // BLOCK)


def work(c):
    if c["kind"] == "norm":
        T, d, w = c["T"], c["d"], _width(c["dtype"])
        return {"bytes": T * d * w * (4 if c["residual"] else 2) + 8 * d + (8 * T if c["stats"] else 0), "flops": 8.0 * T * d}
    if c["kind"] == "dnorm":
        T, d, w = c["T"], c["d"], _width(c["dtype"])
        return {"bytes": T * d * w * (4 if c["residual"] else 3) + 12 * d + 8 * T, "flops": 14.0 * T * d}
    if c["kind"] == "route":
        return {"bytes": 4 * c["T"] * (c["E"] + 2 * c["k"]) + (16 if c["bias"] else 4) * c["E"], "flops": 6.0 * c["T"] * c["E"]}
    if c["kind"] == "droute":
        dense = c["score"] == "softmax" and not c["renorm"]
        return {"bytes": 4 * c["T"] * ((2 if dense else 1) * c["E"] + 4 * c["k"]), "flops": 10.0 * c["T"] * (c["E"] if dense else c["k"])}
    if c["kind"] == "quant":
        # written as codes and scales, which are read and given back as the values that they stand for
        n, w = c["groups"] * c["rows"] * c["n"], _width(c["dtype"])
        return {"bytes": n * (2 * w + 2), "flops": 4.0 * n}
    live = min(c["S"], c["A"])
    if c["kind"] == "product":
        return {"bytes": c["A"] * (c["n"] + c["R"] * _width(c["dtype"])) + live * c["R"] * c["n"], "flops": 2.0 * c["A"] * c["R"] * c["n"]}
    A, d, f = c["A"], c["d"], c["f"]
    return {"bytes": 4 * A * d + (6 * A * f if c["keep"] else 0) + 3 * live * d * f, "flops": 6.0 * A * d * f}


# ---- what a program has in hand before the call

def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"norm": _prepare_norm, "dnorm": _prepare_norm, "route": _prepare_route, "droute": _prepare_route, "quant": _prepare_quant,
         "product": _prepare_product, "experts": _prepare_experts}[case["kind"]](case, g, int(seed))
    s["case"] = case
    return s


def _randn(g, *shape, scale=1.0):
    return torch.randn(*shape, generator=g, device="cuda") * scale


def _context(symi, T, E=1, k=1, d=8, f=8, S=1, dtype="bf16", renorm=1):
    return symi.symi_create(symi.SymiCfg.make(T, E, k, d, f, S, 1, 0, dtype, renorm))


def _prepare_norm(c, g, seed):
    T, d, t = c["T"], c["d"], _type(c["dtype"])
    # a residual stream: rows of different sizes around a mean of their own
    x = (_randn(g, T, d) * torch.exp(_randn(g, T, 1, scale=0.5))).add_(_randn(g, T, 1, scale=0.3)).to(t)
    s = {"X": x, "w": 1 + _randn(g, d, scale=0.1), "b": _randn(g, d, scale=0.1) if c["center"] else None}
    if c["kind"] == "norm":
        s["residual"] = _randn(g, T, d).to(t) if c["residual"] else None
    else:
        x = x.float()
        s["mean"] = x.mean(1) if c["center"] else None
        if c["center"]:
            x -= s["mean"][:, None]
        s["rstd"] = torch.rsqrt(x.square_().mean(1) + EPS)
        s["dY"] = _randn(g, T, d, scale=1e-2).to(t)
        s["dR"] = _randn(g, T, d, scale=1e-2).to(t) if c["residual"] else None
    if own:
        import paper_2504_19925_amd as symi
        s["ctx"] = _context(symi, T, d=d, dtype=c["dtype"])
        s["out"] = torch.empty(T, d, device="cuda", dtype=t)
        if c["kind"] == "norm":
            s["R"] = torch.empty_like(s["out"]) if c["residual"] else None
            s["mean"] = torch.empty(T, device="cuda") if c["stats"] and c["center"] else None
            s["rstd"] = torch.empty(T, device="cuda") if c["stats"] else None
        else:
            s["dw"], s["db"] = torch.empty(d, device="cuda"), torch.empty(d, device="cuda") if c["center"] else None
            s["ws"] = torch.empty(symi.symi_norm_workspace_bytes(s["ctx"]), dtype=torch.uint8, device="cuda")
    return s


def _prepare_route(c, g, seed):
    T, E, k = c["T"], c["E"], c["k"]
    # tokens with a liking of their own, classes of different popularity
    s = {"logits": _randn(g, T, E) + _randn(g, E, scale=0.5), "bias": _randn(g, E, scale=0.05) if c["bias"] else None}
    if c["kind"] == "droute":
        s["idx"], s["gate"] = _choose(s["logits"], s["bias"], c)
        s["dgate"] = _randn(g, T, k)
    if own:
        import paper_2504_19925_amd as symi
        s["ctx"] = _context(symi, T, E, k, S=E, renorm=int(c["renorm"]))
        s["hp"] = symi.SymiScore.make(c["score"], c["groups"], c["top_groups"], c["group_top"], GATE_SCALE)
        if c["kind"] == "route":
            s["idx"], s["gate"] = torch.empty(T, k, dtype=torch.int32, device="cuda"), torch.empty(T, k, device="cuda")
            s["hist"] = torch.empty(E, dtype=torch.int32, device="cuda")
        else:
            s["dlogits"] = torch.empty(T, E, device="cuda")
    return s


def _prepare_quant(c, g, seed):
    G, R, n = c["groups"], c["rows"], c["n"]
    x = torch.empty(G * R, n, device="cuda", dtype=_type(c["dtype"]))
    step = max(1, (1 << 27) // n)
    for r in range(0, G * R, step):     # rows of different sizes, a few columns that stand out
        rows = min(step, G * R - r)
        x[r:r + rows] = _randn(g, rows, n) * torch.exp(_randn(g, rows, 1)) * (1 + 10 * (torch.rand(n, generator=g, device="cuda") < 0.01))
    s = {"X": x.view(G, R, n)}
    if own:
        import paper_2504_19925_amd as symi
        s["ctx"] = _context(symi, 1, dtype=c["dtype"])
        s["q"], s["s"] = _room8(symi, G, R, n, c["block"])
        s["out"] = torch.empty_like(s["X"])
    return s


def _room8(symi, groups, rows, n, block):
    return (torch.empty(groups, rows, symi.symi_pitch8(n), dtype=torch.float8_e4m3fn, device="cuda"),
            torch.empty(groups, -(-rows // block), symi.symi_scale_pitch8(n), dtype=torch.uint8, device="cuda"))


def _codes(x, block):
    """What a program keeps of quantised values [G, R, n]: codes [G, R, p], powers + 127 [G, ceil(R / block), q]; p is n
    up to whole blocks and q the blocks up to whole fours, zeros behind both."""
    G, R, n = x.shape
    q, e = _plain_quant(x, block)
    codes = torch.zeros(G, R, _blocks(n) * BLOCK, device="cuda", dtype=torch.float8_e4m3fn)
    codes[:, :, :n] = q
    s = torch.zeros(G, e.shape[1], -(-_blocks(n) // 4) * 4, device="cuda", dtype=torch.uint8)
    s[:, :, :_blocks(n)] = e.to(torch.uint8)
    return codes, s


def _weights(c, g, R, n):
    """Every slot's weight, in 8 bits; slots in pairs are replicas of one class."""
    codes = torch.empty(c["S"], R, _blocks(n) * BLOCK, device="cuda", dtype=torch.float8_e4m3fn)
    s = torch.empty(c["S"], _blocks(R), -(-_blocks(n) // 4) * 4, device="cuda", dtype=torch.uint8)
    for slot in range(0, c["S"], 2):
        q, e = _codes(_randn(g, 1, R, n, scale=1 / math.sqrt(n)), BLOCK)
        codes[slot:slot + 2], s[slot:slot + 2] = q, e
    return codes, s


def _offsets(c, seed):
    """Where each slot's rows begin: their shares go down with rank ** -skew, in any order."""
    rng = np.random.default_rng(seed)
    p = rng.permutation(np.arange(1, c["S"] + 1) ** -c["skew"])
    at = np.concatenate([[0], np.cumsum(rng.multinomial(c["A"], p / p.sum()))])
    return at.tolist(), torch.from_numpy(at.astype(np.int32)).cuda()


def _prepare_product(c, g, seed):
    A, R, n = c["A"], c["R"], c["n"]
    s = {}
    s["rows"], s["offsets"] = _offsets(c, seed)
    s["a"], s["a_s"] = (x[0] for x in _codes((_randn(g, A, n) * torch.exp(_randn(g, A, 1, scale=0.5)))[None], 1))
    s["w"], s["w_s"] = _weights(c, g, R, n)
    if own:
        import paper_2504_19925_amd as symi
        s["ctx"] = _context(symi, A, c["S"], S=c["S"], dtype=c["dtype"])
        s["Y"] = torch.empty(A, R, device="cuda", dtype=_type(c["dtype"]))
        s["ws"] = torch.empty(symi.symi_workspace8_bytes(s["ctx"]), dtype=torch.uint8, device="cuda")
    return s


def _prepare_experts(c, g, seed):
    A, d, f = c["A"], c["d"], c["f"]
    s = {}
    s["rows"], s["offsets"] = _offsets(c, seed)
    s["X"] = torch.empty(A, d, device="cuda", dtype=torch.bfloat16)
    step = max(1, (1 << 27) // d)
    for r in range(0, A, step):
        s["X"][r:r + step] = _randn(g, min(step, A - r), d)
    s["w1"], s["w1_s"] = _weights(c, g, 2 * f, d)
    s["w2"], s["w2_s"] = _weights(c, g, d, f)
    if own:
        import paper_2504_19925_amd as symi
        s["ctx"] = _context(symi, A, c["S"], d=d, f=f, S=c["S"])
        s["UV"], s["H"] = (torch.empty(A, w, device="cuda", dtype=torch.bfloat16) if c["keep"] else None for w in (2 * f, f))
        s["Y"] = torch.empty(A, d, device="cuda", dtype=torch.bfloat16)
        s["ws"] = torch.empty(symi.symi_workspace8_bytes(s["ctx"]), dtype=torch.uint8, device="cuda")
    return s


# ---- one pass

def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"norm": _own_norm, "dnorm": _own_dnorm, "route": _own_route, "droute": _own_droute, "quant": _own_quant,
                "product": _own_product, "experts": _own_experts}[kind](state)
    return {"norm": _plain_norm, "dnorm": _plain_dnorm, "route": _plain_route, "droute": _plain_droute, "quant": _plain_values,
            "product": _plain_product, "experts": _plain_experts}[kind](state)


def _there(**outputs):
    return {name: x for name, x in outputs.items() if x is not None}


def _own_norm(s):
    import paper_2504_19925_amd as symi
    symi.symi_norm_fwd(s["ctx"], int(s["case"]["center"]), EPS, s["X"], s["residual"], s["w"], s["b"], s["R"], s["out"], s["mean"], s["rstd"])
    return _there(Y=s["out"], R=s["R"], mean=s["mean"], rstd=s["rstd"])


def _own_dnorm(s):
    import paper_2504_19925_amd as symi
    symi.symi_norm_bwd(s["ctx"], int(s["case"]["center"]), s["dY"], s["X"], s["mean"], s["rstd"], s["w"], s["dR"], s["out"], s["dw"], s["db"], s["ws"])
    return _there(dX=s["out"], dw=s["dw"], db=s["db"])


def _own_route(s):
    import paper_2504_19925_amd as symi
    symi.symi_route_scored(s["ctx"], s["hp"], s["logits"], s["bias"], s["idx"], s["gate"], s["hist"])
    if s["bias"] is not None:
        symi.symi_route_bias(s["ctx"], s["hist"], RATE, s["bias"])
    return _there(idx=s["idx"], gate=s["gate"], hist=s["hist"], bias=s["bias"])


def _own_droute(s):
    import paper_2504_19925_amd as symi
    symi.symi_route_scored_bwd(s["ctx"], s["hp"], s["logits"], s["idx"], s["gate"], s["dgate"], s["dlogits"])
    return s["dlogits"]


def _own_quant(s):
    import paper_2504_19925_amd as symi
    c = s["case"]
    symi.symi_quant8(s["ctx"], s["X"], c["groups"], c["rows"], c["n"], c["block"], s["q"], s["s"])
    symi.symi_dequant8(s["ctx"], s["q"], s["s"], c["groups"], c["rows"], c["n"], c["block"], s["out"])
    return s["out"]


def _own_product(s):
    import paper_2504_19925_amd as symi
    symi.symi_product8(s["ctx"], s["a"], s["a_s"], s["offsets"], s["w"], s["w_s"], s["case"]["R"], s["case"]["n"], s["Y"], s["ws"])
    return s["Y"]


def _own_experts(s):
    import paper_2504_19925_amd as symi
    symi.symi_expert_fwd8(s["ctx"], s["X"], s["offsets"], s["w1"], s["w1_s"], s["w2"], s["w2_s"], s["UV"], s["H"], s["Y"], s["ws"])
    return _there(Y=s["Y"], UV=s["UV"], H=s["H"])


def _plain_norm(s):
    c, r = s["case"], s["X"].float()
    out = None
    if s["residual"] is not None:
        out = (r + s["residual"].float()).to(s["X"].dtype)
        r = out.float()
    mean = None
    if c["center"]:
        mean = r.mean(1)
        r = r - mean[:, None]
    rstd = torch.rsqrt((r * r).mean(1) + EPS)
    y = r * rstd[:, None] * s["w"]
    if s["b"] is not None:
        y += s["b"]
    y = y.to(s["X"].dtype)
    return _there(Y=y, R=out, mean=mean if c["stats"] else None, rstd=rstd if c["stats"] else None)


def _plain_dnorm(s):
    x, dy = s["X"].float(), s["dY"].float()
    if s["case"]["center"]:
        x = x - s["mean"][:, None]
    x = x * s["rstd"][:, None]
    dw = (dy * x).sum(0)
    db = dy.sum(0) if s["case"]["center"] else None
    g = dy * s["w"]
    dx = g - x * (g * x).mean(1, keepdim=True)
    if s["case"]["center"]:
        dx -= g.mean(1, keepdim=True)
    dx *= s["rstd"][:, None]
    if s["dR"] is not None:
        dx += s["dR"].float()
    return _there(dX=dx.to(s["X"].dtype), dw=dw, db=db)


def _choose(logits, bias, c):
    """(idx [T, k], gate [T, k]).  Classes are compared in 64 bits."""
    T, E = logits.shape
    z = logits.double()
    if c["score"] == "sigmoid":
        score = 1 / (1 + torch.exp(-z))
    else:
        score = torch.exp(z - z.amax(1, keepdim=True))
        score = score / score.sum(1, keepdim=True)
    by = z if bias is None else score + bias.double()
    if c["groups"] > 1:
        top = min(c["group_top"], E // c["groups"])
        of_group = (score if bias is None and top > 1 else by).view(T, c["groups"], -1)
        of_group = torch.sort(of_group, dim=2, descending=True)[0][:, :, :top].sum(2)
        kept = torch.sort(of_group, dim=1, descending=True, stable=True)[1][:, :c["top_groups"]]
        live = torch.zeros_like(of_group, dtype=torch.bool).scatter_(1, kept, True)
        by = torch.where(live[:, :, None], by.view(T, c["groups"], -1), -math.inf).view(T, E)
    idx = torch.sort(by, dim=1, descending=True, stable=True)[1][:, :c["k"]]
    gate = score.gather(1, idx)
    if c["renorm"]:
        gate = gate / gate.sum(1, keepdim=True)
    return idx.to(torch.int32), (gate * GATE_SCALE).float()


def _plain_route(s):
    c = s["case"]
    idx, gate = _choose(s["logits"], s["bias"], c)
    hist = torch.zeros(c["E"], dtype=torch.int32, device="cuda")
    hist.index_add_(0, idx.view(-1).long(), torch.ones_like(idx.view(-1)))
    if s["bias"] is not None:
        s["bias"] += RATE * torch.sign(c["T"] * c["k"] - c["E"] * hist.long())
    return _there(idx=idx, gate=gate, hist=hist, bias=s["bias"])


def _plain_droute(s):
    c, idx = s["case"], s["idx"].long()
    z = s["logits"]
    g = s["gate"] / GATE_SCALE
    dg = s["dgate"] * GATE_SCALE
    out = torch.zeros_like(z)
    if c["renorm"]:
        dz = g * (dg - (g * dg).sum(1, keepdim=True))
        if c["score"] == "sigmoid":
            dz = dz / (1 + torch.exp(z.gather(1, idx)))
        return out.scatter_(1, idx, dz)
    if c["score"] == "sigmoid":
        return out.scatter_(1, idx, dg * g / (1 + torch.exp(z.gather(1, idx))))
    p = torch.exp(z - z.amax(1, keepdim=True))
    p = p / p.sum(1, keepdim=True)
    return p * (out.scatter_(1, idx, dg) - (g * dg).sum(1, keepdim=True))


def _share(e, rows, n, block):
    """The scale of every value: 2 ** (e - 127), as numbers [G, rows, n]."""
    scale = torch.where(e > 0, e << 23, 1 << 22).to(torch.int32).view(torch.float32)     # as a number's bits; 2 ** -127 is a denormal one
    scale = scale.repeat_interleave(BLOCK, 2)[:, :, :n]
    return scale if block == 1 else scale.repeat_interleave(block, 1)[:, :rows]


def _plain_quant(x, block):
    """Codes in e4m3 and powers + 127 of [G, R, n]."""
    G, R, n = x.shape
    x = x.float()
    pad = torch.nn.functional.pad(x.abs(), (0, -n % BLOCK, 0, -R % block))
    most = pad.view(G, -(-R // block), block, _blocks(n), BLOCK).amax((2, 4))
    # the smallest power of two with which the largest value is at most 448 = 1.75 * 2 ** 8
    e = ((most.view(torch.int32) + 0x1fffff) >> 23).sub_(8).clamp_(min=0)
    return (x / _share(e, R, n, block)).to(torch.float8_e4m3fn), e


def _plain_values(s):
    c = s["case"]
    q, e = _plain_quant(s["X"], c["block"])
    return (q.float() * _share(e, c["rows"], c["n"], c["block"])).to(s["X"].dtype)


def _of_slot(w, s, slot):
    return w[slot].float() * _share(s[slot:slot + 1, :, :_blocks(w.shape[2])].int(), w.shape[1], w.shape[2], BLOCK)[0]


def _plain_product(s):
    at = s["rows"]
    a = s["a"].float() * _share(s["a_s"][None, :, :_blocks(s["case"]["n"])].int(), 0, s["a"].shape[1], 1)[0]
    return torch.cat([a[at[q]:at[q + 1]] @ _of_slot(s["w"], s["w_s"], q).t() for q in range(s["case"]["S"])]).to(_type(s["case"]["dtype"]))


def _back(x):
    """The values that rows have in 8 bits, in single precision."""
    q, e = _plain_quant(x[None], 1)
    return (q.float() * _share(e, 0, x.shape[1], 1))[0]


def _plain_slot(s, q):
    d, f = s["case"]["d"], s["case"]["f"]
    uv = _back(s["X"][s["rows"][q]:s["rows"][q + 1]]) @ _of_slot(s["w1"], s["w1_s"], q)[:, :d].t()
    u = uv[:, :f]
    h = u / (1 + torch.exp(-u)) * uv[:, f:]
    y = _back(h) @ _of_slot(s["w2"], s["w2_s"], q)[:, :f].t()
    return [x.to(torch.bfloat16) for x in ((y, uv, h) if s["case"]["keep"] else (y,))]


def _plain_experts(s):
    parts = zip(*[_plain_slot(s, q) for q in range(s["case"]["S"])])
    return dict(zip(("Y", "UV", "H"), (torch.cat(p) for p in parts)))


# ---- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "dnorm": _exact_dnorm, "route": _exact_route, "droute": _exact_droute, "quant": _exact_quant,
            "product": _exact_product, "experts": _exact_experts}[case["kind"]](s, case)


def _exact_norm(s, c):
    r, out = s["X"].double(), None
    if c["residual"]:
        out = s["X"].double() + s["residual"].double()
        r = out.to(s["X"].dtype).double()      # the norm is that of the sum as it is kept
    if c["center"]:
        var, mean = torch.var_mean(r, 1, correction=0)
    else:
        var, mean = r.square().mean(1), torch.zeros(c["T"], device="cuda", dtype=torch.float64)
    y = (r - mean[:, None]) / (var + EPS).sqrt()[:, None] * s["w"].double()
    if s["b"] is not None:
        y = y + s["b"].double()
    return _there(Y=y, R=out, mean=mean if c["stats"] and c["center"] else None, rstd=1 / (var + EPS).sqrt() if c["stats"] else None)


def _exact_dnorm(s, c):
    T, d = c["T"], c["d"]
    dx = torch.empty(T, d, device="cuda", dtype=torch.float64)
    dw, db = torch.zeros(d, device="cuda", dtype=torch.float64), torch.zeros(d, device="cuda", dtype=torch.float64)
    for r in range(0, T, 4096):
        rows = slice(r, min(T, r + 4096))
        dy, rstd = s["dY"][rows].double(), s["rstd"][rows].double()[:, None]
        x = s["X"][rows].double()
        x = (x - s["mean"][rows].double()[:, None] if c["center"] else x) * rstd
        dw += torch.einsum("td,td->d", dy, x)
        db += dy.sum(0)
        g = dy * s["w"].double()
        along = (g * x).sum(1, keepdim=True) / d
        level = g.sum(1, keepdim=True) / d if c["center"] else 0.0
        dx[rows] = (g - level - x * along) * rstd + (s["dR"][rows].double() if c["residual"] else 0.0)
    return _there(dX=dx, dw=dw, db=db if c["center"] else None)


def _exact_route(s, c):
    T, E, k, G = c["T"], c["E"], c["k"], c["groups"]
    z = s["logits"].double().cpu().numpy()
    if c["score"] == "sigmoid":
        score = np.exp(-np.logaddexp(0, -z))
    else:
        top = z.max(1, keepdims=True)
        score = np.exp(z - top - np.log(np.exp(z - top).sum(1, keepdims=True)))
    by = score + s["bias"].double().cpu().numpy() if c["bias"] else score
    if G > 1:
        most = -np.sort(-by.reshape(T, G, -1), axis=2)[:, :, :c["group_top"]]
        worst = np.argsort(-most.sum(2), axis=1, kind="stable")[:, c["top_groups"]:]
        by = by.reshape(T, G, -1).copy()
        np.put_along_axis(by, worst[:, :, None], -np.inf, 1)
        by = by.reshape(T, E)
    idx = np.argsort(-by, axis=1, kind="stable")[:, :k]
    gate = np.take_along_axis(score, idx, 1)
    if c["renorm"]:
        gate = gate / gate.sum(1, keepdims=True)
    hist = np.bincount(idx.reshape(-1), minlength=E)
    bias = None
    if c["bias"]:
        bias = s["bias"].double() + RATE * torch.from_numpy(np.sign(T * k / E - hist)).cuda()
    return _there(idx=torch.from_numpy(idx.astype(np.int32)).cuda(), gate=torch.from_numpy(gate * GATE_SCALE).cuda(),
                  hist=torch.from_numpy(hist.astype(np.int32)).cuda(), bias=bias)


def _exact_droute(s, c):
    z = s["logits"].double().requires_grad_()
    if c["score"] == "sigmoid":
        gate = torch.sigmoid(z).gather(1, s["idx"].long())
    else:
        gate = torch.softmax(z, 1).gather(1, s["idx"].long())
    if c["renorm"]:
        gate = gate / gate.sum(1, keepdim=True)
    (gate * GATE_SCALE * s["dgate"].double()).sum().backward()
    return z.grad


def _two_to(e):
    """2 ** e in 64 bits, exactly."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _near(x, block):
    """x [R, n] in 64 bits to the values that it has in 8: multiples of 2 ** (exponent - 3), of 2 ** -9 at the least, next
    to a largest one of at most 448."""
    R, n = x.shape
    out = torch.zeros(-(-R // block) * block, _blocks(n) * BLOCK, device="cuda", dtype=torch.float64)
    out[:R, :n] = x
    out = out.view(-1, block, _blocks(n), BLOCK)
    most = out.abs().amax((1, 3), keepdim=True)
    e = torch.ceil(torch.log2(most / TOP)).clamp(min=-127)
    e = torch.where(TOP * _two_to(e - 1) >= most, e - 1, e).clamp(min=-127)   # where the logarithm was rounded up
    scale = _two_to(e)
    y = out / scale
    step = _two_to((torch.frexp(y)[1] - 1).clamp(min=-6) - 3)
    return (torch.round(y / step) * step * scale).reshape(-1, _blocks(n) * BLOCK)[:R, :n]


def _exact_quant(s, c):
    return torch.stack([_near(x.double(), c["block"]) for x in s["X"]]) if c["block"] > 1 else _near(s["X"][0].double(), 1)[None]


def _value(codes, powers, slot, n):
    R = codes.shape[1]
    e = powers[slot].long()[torch.arange(R, device="cuda") // BLOCK][:, torch.arange(n, device="cuda") // BLOCK]
    return codes[slot, :, :n].double() * _two_to(e - 127)


def _exact_product(s, c):
    n = c["n"]
    e = s["a_s"].long()[:, torch.arange(n, device="cuda") // BLOCK]
    a = s["a"][:, :n].double() * _two_to(e - 127)
    out = torch.empty(c["A"], c["R"], device="cuda", dtype=torch.float64)
    for q in range(c["S"]):
        rows = slice(s["rows"][q], s["rows"][q + 1])
        out[rows] = a[rows] @ _value(s["w"], s["w_s"], q, n).t()
    return out


def _exact_experts(s, c):
    A, d, f = c["A"], c["d"], c["f"]
    new = lambda w: torch.empty(A, w, device="cuda", dtype=torch.float64)   # noqa: E731
    out = {"Y": new(d)} | ({"UV": new(2 * f), "H": new(f)} if c["keep"] else {})
    for q in range(c["S"]):
        rows = slice(s["rows"][q], s["rows"][q + 1])
        if rows.start == rows.stop:
            continue
        uv = _near(s["X"][rows].double(), 1) @ _value(s["w1"], s["w1_s"], q, d).t()
        h = uv[:, :f] * torch.sigmoid(uv[:, :f]) * uv[:, f:]
        out["Y"][rows] = _near(h, 1) @ _value(s["w2"], s["w2_s"], q, f).t()
        if c["keep"]:
            out["UV"][rows], out["H"][rows] = uv, h
    return out
