"""The two ends of a training step around the MoE layers, as cases that can be measured: token embedding and its
gradient, the clipped policy loss from logits, and AdamW over the tensors that are no experts.

`run` is one call (one optimizer step) on what a training program holds: in elementary torch operations where `own` is
false, through the library where it is true.  Sizes are those of workloads/configs.py (c1 .. c5) with vocabularies
from 8000 to 131072 and ragged ones between them.

kinds   embed    X[t] = scale * table[tokens[t]], tokens outside the table (padding) give zero rows
        table    its gradient: dTable[v] = scale * sum of dX[t] over the tokens t that are v; `add`: added to the table's
                 gradient from the other uses of the table (tied weights, micro-batches)
        policy   rows of logits to mode "logp": log probabilities of the tokens taken; "loss": with the clipped
                 policy loss and its KL term; "grad": with the gradient of the logits
        adamw    one step over all tensors, states in `bits` bits per value
"""
import itertools
import math

import numpy as np
import torch

own = False

CLIP_LOW, CLIP_HIGH, KL_COEF = 0.2, 0.28, 0.04
LR, BETA1, BETA2, EPS, DECAY = (float(np.float32(x)) for x in (1e-3, 0.9, 0.999, 1e-8, 0.1))
BLOCK = 256                    # values that share one scale of an 8-bit state
SEQ = 512                      # tokens of one sequence of a policy batch; its first ones are the prompt
SMALLEST = float(np.finfo(np.float32).tiny)
LARGEST = float(np.finfo(np.float32).max)
M_UNIT = float(np.float32(1.0 / 127 ** 2))
V_UNIT = float(np.float32(1.0 / 255 ** 2))
WORD = 0xffffffff


def _embed(kind, dtype, T, d, V, zipf=1.0, pad=0.0, add=False):
    return {"kind": kind, "dtype": dtype, "T": T, "d": d, "V": V, "zipf": zipf, "pad": pad, "add": add}


def _policy(mode, dtype, T, V, ld=0, masked=0.0, tau=1.0, kl=True):
    return {"kind": "policy", "mode": mode, "dtype": dtype, "T": T, "V": V, "ld": ld or V, "masked": masked, "tau": tau,
            "kl": kl}


def _adamw(bits, layers, d, E, dense, V, param="f32", grad="f32"):
    """`layers` times the gate network [E, d] with its bias, two norms and `dense` matrices [d, d]; a table [V, d]."""
    return {"kind": "adamw", "bits": bits, "layers": layers, "d": d, "E": E, "dense": dense, "V": V, "param": param,
            "grad": grad}


def listed():
    named = [
        # c5's batch at the bottom of the model: half a gigabyte of rows out of a gigabyte of table
        ("c5 embedding", _embed("embed", "bf16", 65536, 4096, 131072, pad=0.05)),
        # c1, the smallest model that anybody trains: latency
        ("c1 table gradient", _embed("table", "f32", 1024, 128, 8000)),
        # c2's batch with the table tied to the output product, whose gradient is there already; ragged vocabulary
        ("c2 tied table gradient", _embed("table", "bf16", 8192, 1024, 50001, zipf=1.1, pad=0.1, add=True)),
        # c5's batch: a gigabyte of gradient, a few tokens that come thousands of times
        ("c5 table gradient", _embed("table", "bf16", 65536, 4096, 65536)),
        # a serving process that reports log probabilities: a few tokens
        ("logp of 16 tokens", _policy("logp", "bf16", 16, 128000)),
        # the loss of c2's batch in validation: prompts masked, vocabulary padded to whole tiles
        ("c2 policy loss", _policy("loss", "bf16", 8192, 50001, ld=50048, masked=0.4)),
        # a single-precision run, rows that start anywhere, sampled at a temperature
        ("ragged policy step f32", _policy("grad", "f32", 777, 32003, masked=0.2, tau=0.7)),
        # c3's batch with the largest vocabulary
        ("c3 policy step", _policy("grad", "bf16", 16384, 131072, masked=0.25)),
        # the gate network of c1 with its norms: launches only
        ("c1 gate step", _adamw(32, 1, 128, 8, 0, 0)),
        # c4's dense part, bf16 weights with their fp32 masters
        ("c4 step", _adamw(32, 4, 2048, 64, 4, 65536, param="bf16")),
        # odd widths: every tensor ends inside a block, gradients in bf16 as a matrix product leaves them
        ("ragged 8-bit step", _adamw(8, 6, 1001, 13, 3, 8191, grad="bf16")),
        # c5's dense part, states in 8 bits
        ("c5 8-bit step", _adamw(8, 4, 4096, 128, 4, 65536)),
    ]
    return [dict(c, name=name) for name, c in named]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    kind = rng.choice(("embed", "table", "table", "policy", "policy", "policy", "adamw", "adamw"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if kind in ("embed", "table"):
        d, T, V = 8 * round(_log(rng, 1, 512)), round(_log(rng, 1, 65536)), round(_log(rng, 300, 131072))
        return _embed(kind, dtype, min(T, (1 << 28) // d), d, min(V, (1 << 28) // d), zipf=rng.choice((0.0, 0.7, 1.0, 1.3)),
                      pad=rng.choice((0.0, 0.0, 0.1, 0.5)), add=kind == "table" and rng.random() < 0.5)
    if kind == "policy":
        V = round(_log(rng, 1000, 262144))
        T = min(round(_log(rng, 1, 16384)), (1 << (31 if dtype == "bf16" else 30)) // (V + 64))
        mode = rng.choice(("logp", "loss", "grad", "grad"))
        return _policy(mode, dtype, T, V, ld=rng.choice((V, -(-V // 64) * 64)), masked=rng.choice((0.0, 0.0, 0.3, 0.6)),
                       tau=rng.choice((1.0, 1.0, 0.6)), kl=mode != "logp" and rng.random() < 0.7)
    d = round(_log(rng, 16, 4096))
    return _adamw(rng.choice((8, 8, 32)), rng.randint(1, 32 if d < 1024 else 4), d, rng.choice((4, 8, 13, 64, 128)), rng.randint(0, 4),
                  rng.choice((0, 1, 1)) * min(round(_log(rng, 300, 65536)), (1 << 27) // d),
                  param=rng.choice(("f32", "bf16")), grad=rng.choice(("f32", "f32", "bf16")))


# ---- sizes and work

def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _width(name):
    return 2 if name == "bf16" else 4


def _share(c):
    """How likely each row of the table is: rank^-zipf."""
    p = np.arange(1, c["V"] + 1, dtype=np.float64) ** -c["zipf"]
    return p / p.sum()


def _masked_rows(c):
    """Rows of a policy batch that belong to a prompt: the first ones of every sequence."""
    whole, rest = divmod(c["T"], SEQ)
    return whole * int(c["masked"] * SEQ) + int(c["masked"] * rest)


def _layout(c):
    """The lengths of the tensors of an optimizer step, whether they decay, and where each starts in the flat buffers: at whole blocks."""
    d, layer = c["d"], [(c["E"] * c["d"], 1.0), (c["E"], 0.0), (c["d"], 0.0), (c["d"], 0.0)] + [(c["d"] ** 2, 1.0)] * c["dense"]
    tensors = layer * c["layers"] + ([(c["V"] * d, 1.0)] if c["V"] else [])
    blocks = [-(-n // BLOCK) for n, _ in tensors]
    ends = list(itertools.accumulate(blocks))
    return [(n, decay, (end - b) * BLOCK) for (n, decay), b, end in zip(tensors, blocks, ends)], ends[-1]


def work(c):
    if c["kind"] in ("embed", "table"):
        w, rows = _width(c["dtype"]), c["T"] * (1 - c["pad"])
        distinct = float((-np.expm1(rows * np.log1p(-np.minimum(_share(c), 1 - 1e-12)))).sum())
        if c["kind"] == "embed":
            return {"bytes": 4 * c["T"] + (distinct + c["T"]) * c["d"] * w, "flops": rows * c["d"]}
        return {"bytes": 4 * c["T"] + rows * c["d"] * w + 4 * c["d"] * (2 * distinct if c["add"] else c["V"]),
                "flops": rows * c["d"]}
    if c["kind"] == "policy":
        w, rows = _width(c["dtype"]), c["T"] - _masked_rows(c)
        grad = c["T"] * c["ld"] * w if c["mode"] == "grad" else 0
        return {"bytes": rows * c["V"] * w + grad + (12 if c["mode"] == "logp" else 28) * c["T"],
                "flops": rows * c["V"] * (8.0 if grad else 5.0)}
    n = sum(t[0] for t in _layout(c)[0])
    param = 10 if c["param"] == "bf16" else 8
    # the 8-bit states are read, written, and given back as the values that they stand for
    states = 16 if c["bits"] == 32 else 4 + 16 / BLOCK + 8
    return {"bytes": n * (_width(c["grad"]) + param + states), "flops": n * (15.0 if c["bits"] == 32 else 60.0)}


# ---- what a program has in hand before the call

def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"embed": _prepare_rows, "table": _prepare_rows, "policy": _prepare_policy, "adamw": _prepare_adamw}[case["kind"]](case, g)
    s["case"] = case
    return s


def _randn(g, *shape, scale=1.0):
    return torch.randn(*shape, generator=g, device="cuda") * scale


def _rand(g, *shape):
    return torch.rand(*shape, generator=g, device="cuda")


def _context(symi, T, d, dtype):
    return symi.symi_create(symi.SymiCfg.make(T, 1, 1, d, 8, 1, 1, 0, dtype))


def _prepare_rows(c, g):
    T, d, V = c["T"], c["d"], c["V"]
    at = torch.searchsorted(torch.from_numpy(np.cumsum(_share(c))).cuda(), torch.rand(T, generator=g, device="cuda", dtype=torch.float64))
    tokens = torch.where(_rand(g, T) < c["pad"], -1, at.clamp(max=V - 1)).to(torch.int32)
    s = {"tokens": tokens, "scale": float(np.float32(math.sqrt(d)))}
    if c["kind"] == "embed":
        s["table"] = _randn(g, V, d, scale=0.02).to(_type(c["dtype"]))
        s["X"] = torch.empty(T, d, device="cuda", dtype=_type(c["dtype"]))
    else:
        s["dX"] = _randn(g, T, d).to(_type(c["dtype"]))
        s["dTable"] = _randn(g, V, d) if c["add"] else torch.empty(V, d, device="cuda")
    if own:
        import paper_2504_19925_amd as symi
        s["ctx"] = _context(symi, T, d, c["dtype"])
        if c["kind"] == "table":
            s["ws"] = torch.empty(symi.symi_embed_workspace_bytes(s["ctx"], V), dtype=torch.uint8, device="cuda")
    return s


def _prepare_policy(c, g):
    T, V, ld = c["T"], c["V"], c["ld"]
    logits = torch.empty(T, ld, device="cuda", dtype=_type(c["dtype"]))
    logp = torch.empty(T, device="cuda")
    action = torch.empty(T, device="cuda", dtype=torch.int32)
    step = max(1, (1 << 27) // ld)
    for r in range(0, T, step):   # flat and peaked rows; the tokens taken are sampled from them
        z = _randn(g, min(step, T - r), ld) * (1.0 + 4.0 * _rand(g, min(step, T - r), 1))
        logits[r:r + step] = z.to(logits.dtype)
        z = logits[r:r + step, :V].float() / c["tau"]
        noise = -torch.log(-torch.log(_rand(g, *z.shape).clamp_(1e-9, 1 - 1e-7)))
        action[r:r + step] = noise.add_(z).argmax(1).to(torch.int32)
        logp[r:r + step] = (z.gather(1, action[r:r + step, None].long())[:, 0] - torch.logsumexp(z, 1))
    # probability ratios of a policy a few updates on; where the loss has its kinks, rounding decides on which side a
    # token is, so none is nearer to one than 1e-3
    ratio = torch.exp(0.15 * _randn(g, T))
    for kink in (1 - CLIP_LOW, 1 + CLIP_HIGH):
        ratio = torch.where((ratio - kink).abs() < 1e-3, kink + 2e-3, ratio)
    place = torch.arange(T, device="cuda")
    length = (T - place // SEQ * SEQ).clamp(max=SEQ)   # of the token's sequence
    taken = (place % SEQ >= torch.floor(c["masked"] * length.double())).float()
    s = {"logits": logits, "action": action, "old": logp - torch.log(ratio), "ref": logp + 0.1 * _randn(g, T) if c["kl"] else None,
         "advantage": _randn(g, T), "weight": taken / taken.sum().clamp(min=1)}
    if own:
        import paper_2504_19925_amd as symi
        s["ctx"] = _context(symi, T, 8, c["dtype"])
        s["hp"] = symi.SymiPolicy.make(CLIP_LOW, CLIP_HIGH, KL_COEF if c["kl"] else 0.0, temperature=c["tau"], dtype=c["dtype"])
        s["ws"] = torch.empty(symi.symi_policy_workspace_bytes(s["ctx"]), dtype=torch.uint8, device="cuda")
        s["logp"], s["stats"] = torch.empty(T, device="cuda"), torch.empty(4, device="cuda")
        s["dlogits"] = torch.empty_like(logits) if c["mode"] == "grad" else None
    return s


def _prepare_adamw(c, g):
    tensors, blocks = _layout(c)
    n = blocks * BLOCK
    inside = torch.zeros(n, dtype=torch.bool, device="cuda")
    for size, _, start in tensors:
        inside[start:start + size] = True
    # gradients whose size differs from block to block; rows of the table that no token chose have none
    size = torch.exp(_randn(g, blocks, 1)) * (_rand(g, blocks, 1) > 0.1)
    w = (_randn(g, n) * 0.02).mul_(inside)
    grad = (_randn(g, blocks, BLOCK) * size * 1e-3).view(-1).mul_(inside).to(_type(c["grad"]))
    m = (_randn(g, blocks, BLOCK) * size * 3e-4).view(-1).mul_(inside)
    v = (_randn(g, blocks, BLOCK) * size * 1e-3).square_().view(-1).mul_(inside)
    s = {"step": 100, "seed": 12345, "clip": torch.full((1,), 0.37, device="cuda"), "grad": grad, "m": m, "v": v,
         "w": w, "param": w.to(torch.bfloat16) if c["param"] == "bf16" else None,
         "decay": torch.repeat_interleave(torch.tensor([t[1] for t in tensors], device="cuda"),
                                          torch.tensor([-(-t[0] // BLOCK) for t in tensors], device="cuda"))[:, None]}
    if c["bits"] == 8:
        m, v = m.view(blocks, BLOCK), v.view(blocks, BLOCK)
        s["m_scale"], s["v_scale"] = m.abs().amax(1), v.amax(1)
        s["m"] = (127 * (m.abs() / s["m_scale"][:, None].clamp(min=SMALLEST)).sqrt()).round().mul(m.sign()).to(torch.int8).view(-1)
        s["v"] = (255 * (v / s["v_scale"][:, None].clamp(min=SMALLEST)).sqrt().sqrt()).ceil().clamp(max=255).to(torch.uint8).view(-1)
        del m, v
    if own:
        import paper_2504_19925_amd as symi
        s["ctx"] = _context(symi, 1, 8, "f32")
        if c["bits"] == 8:
            s["m_value"], s["v_value"] = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
        s["opt"] = symi.symi_adamw_create([_tensor(s, c, t) for t in tensors])
    return s


def _tensor(s, c, t):
    """One tensor of the step, as the library takes it: its part of the flat buffers."""
    n, decay, start = t
    at, block = slice(start, start + n), slice(start // BLOCK, start // BLOCK - (-n // BLOCK))
    half, codes = c["param"] == "bf16", c["bits"] == 8
    return {"param": s["param"][at] if half else s["w"][at], "master": s["w"][at] if half else None, "grad": s["grad"][at],
            "m": s["m"][at], "v": s["v"][at], "m_scale": s["m_scale"][block] if codes else None,
            "v_scale": s["v_scale"][block] if codes else None, "decay": decay}


# ---- one pass

def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"embed": _own_embed, "table": _own_table, "policy": _own_policy, "adamw": _own_adamw}[kind](state)
    return {"embed": _plain_embed, "table": _plain_table, "policy": _plain_policy, "adamw": _plain_adamw}[kind](state)


def _own_embed(s):
    import paper_2504_19925_amd as symi
    symi.symi_embed_fwd(s["ctx"], s["tokens"], s["table"], s["case"]["V"], s["scale"], s["X"])
    return s["X"]


def _own_table(s):
    import paper_2504_19925_amd as symi
    symi.symi_embed_bwd(s["ctx"], s["tokens"], s["dX"], s["case"]["V"], s["scale"], int(s["case"]["add"]), s["dTable"], s["ws"])
    return s["dTable"]


def _own_policy(s):
    import paper_2504_19925_amd as symi
    c = s["case"]
    if c["mode"] == "logp":
        symi.symi_token_logp(s["ctx"], s["hp"], s["logits"], c["V"], c["ld"], s["action"], s["weight"], s["logp"])
        return s["logp"]
    symi.symi_policy_loss(s["ctx"], s["hp"], s["logits"], c["V"], c["ld"], s["action"], s["old"], s["ref"], s["advantage"],
                          s["weight"], s["logp"], s["stats"], s["dlogits"], s["ws"])
    return {"logp": s["logp"], "stats": s["stats"]} | ({"dlogits": s["dlogits"]} if c["mode"] == "grad" else {})


def _own_adamw(s):
    import paper_2504_19925_amd as symi
    s["step"] += 1
    symi.symi_adamw_step(s["ctx"], s["opt"], symi.SymiAdam(LR, BETA1, BETA2, EPS, DECAY, 1.0, s["step"]), s["clip"], s["seed"])
    m, v = s["m"], s["v"]
    if s["case"]["bits"] == 8:
        m, v = s["m_value"], s["v_value"]
        symi.symi_adamw_decode(s["ctx"], s["opt"], m, v)
    return {"w": s["w"], "m": m, "v": v} | ({"param": s["param"]} if s["param"] is not None else {})


def _plain_embed(s):
    V = s["case"]["V"]
    inside = (s["tokens"] >= 0) & (s["tokens"] < V)
    rows = s["table"][s["tokens"].long().clamp(0, V - 1)].float() * s["scale"]
    return torch.where(inside[:, None], rows, 0.0).to(s["table"].dtype)


def _plain_table(s):
    V, d = s["case"]["V"], s["case"]["d"]
    at = torch.where((s["tokens"] >= 0) & (s["tokens"] < V), s["tokens"], V).long()
    out = torch.zeros(V + 1, d, device="cuda").index_add_(0, at, s["dX"].float() * s["scale"])[:V]
    if not s["case"]["add"]:
        return out
    s["dTable"] += out
    return s["dTable"]


def _plain_policy(s):
    c = s["case"]
    T, V, w = c["T"], c["V"], s["weight"]
    y = s["action"].long()
    active = (w != 0) & (y >= 0) & (y < V)
    y = y.clamp(0, V - 1)[:, None]
    z = s["logits"][:, :V].float() * float(np.float32(1 / c["tau"]))
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    lp = torch.where(active, ((z.gather(1, y) - top) - torch.log(total))[:, 0], 0.0)
    if c["mode"] == "logp":
        return lp
    A, ratio = s["advantage"], torch.exp(lp - s["old"])
    clipped = ((A > 0) & (ratio > 1 + CLIP_HIGH)) | ((A < 0) & (ratio < 1 - CLIP_LOW))
    w = torch.where(active, w, 0.0)
    gain = -A * torch.where(clipped, torch.where(A > 0, 1 + CLIP_HIGH, 1 - CLIP_LOW), ratio)
    slope = -torch.where(clipped, 0.0, A * ratio)
    kl = torch.zeros_like(gain)
    if c["kl"]:
        far = s["ref"] - lp
        kl = torch.expm1(far) - far
        slope = slope - KL_COEF * torch.expm1(far)
    stats = torch.stack([(w * (gain + KL_COEF * kl)).sum(), (w * gain).sum(), (w * kl).sum(), (w * clipped).sum()])
    if c["mode"] == "loss":
        return {"logp": lp, "stats": stats}
    slope = (w * slope * float(np.float32(1 / c["tau"])))[:, None]
    dz = torch.zeros(T, c["ld"], device="cuda")
    dz[:, :V] = e.div_(total).mul_(-slope).scatter_add_(1, y, slope)
    return {"logp": lp, "stats": stats, "dlogits": dz.to(s["logits"].dtype)}


def _mix(x):
    x = x ^ (x >> 16)
    x = x * 0xBB67AE85 & WORD
    x = x ^ (x >> 15)
    x = x * 0x6A09E667 & WORD
    return x ^ (x >> 16)


def _random(s, blocks):
    """Two numbers in (0, 1) of 16 bits for every value, from the seed, the step and the value's place."""
    key = _mix((_mix(s["seed"] & WORD) + s["step"]) & WORD)
    i = torch.arange(blocks * BLOCK, device="cuda").view(blocks, BLOCK)
    times = torch.tensor([0x3C6EF373, 0xA54FF53B, 0x510E527F, 0x9B05688D], device="cuda")[i & 3]
    r = _mix((i >> 2) * 0x9E3779B1 + key & WORD) * times & WORD
    r = r ^ (r >> 15)
    return ((r & 0xffff).float() + 0.5) * 2.0 ** -16, ((r >> 16).float() + 0.5) * 2.0 ** -16


def _m_of(code, a):
    return code * code * M_UNIT * a


def _v_of(code, a):
    q = code * code * V_UNIT
    return q * q * a


def _scale_of(x):
    """The largest of each block; 0 for a block of nothing but denormal numbers, NaN for one that is not finite."""
    a = x.amax(1, keepdim=True)
    return torch.where(a < SMALLEST, 0.0, torch.where(a <= LARGEST, a, math.nan))


def _between(x, a, guess, top, of, u):
    """Code of x: one of its two neighbours in value, the upper one as often as x is near to it."""
    lo = guess.floor().clamp(0, top - 1)
    lo = lo - (of(lo, a) > x).float()
    lo = (lo + (of(lo + 1, a) <= x).float()).clamp(0, top - 1)
    below, above = of(lo, a), of(lo + 1, a)
    code = lo + (x - below > u * (above - below)).float()
    return torch.where((a >= SMALLEST) & (a <= LARGEST), code, 0.0)


def _plain_adamw(s):
    c, blocks = s["case"], s["decay"].shape[0]
    s["step"] += 1
    one = np.float32(1)
    keep1, keep2 = float(one - np.float32(BETA1)), float(one - np.float32(BETA2))
    fix1, fix2 = (float(np.float32(1 / (1 - b ** s["step"]))) for b in (BETA1, BETA2))
    g = s["grad"].view(blocks, BLOCK).float() * s["clip"]
    m, v = s["m"].view(blocks, BLOCK), s["v"].view(blocks, BLOCK)
    if c["bits"] == 8:
        m, v = m.float(), v.float()
        m = _m_of(m.abs(), s["m_scale"][:, None]) * m.sign()
        v = _v_of(v, s["v_scale"][:, None])
    m = m * BETA1 + g * keep1
    v = v * BETA2 + (g * keep2) * g
    w = s["w"].view(blocks, BLOCK)
    w -= LR * ((m * fix1) / ((v * fix2).sqrt() + EPS) + (s["decay"] * DECAY) * w)
    if c["bits"] == 8:
        u_m, u_v = _random(s, blocks)
        a, x = _scale_of(m.abs()), m.abs()
        code = _between(x, a, 127 * (x / a).sqrt(), 127, _m_of, u_m) * m.sign()
        s["m"].copy_(code.view(-1))
        s["m_scale"].copy_(a[:, 0])
        m = _m_of(code.abs(), a) * code.sign()
        a = _scale_of(v)
        code = _between(v, a, 255 * (v / a).sqrt().sqrt(), 255, _v_of, u_v)
        code = torch.where((v > 0) & (a > 0), code.clamp(min=1), code)   # 0 stands for no gradient ever
        s["v"].copy_(code.view(-1))
        s["v_scale"].copy_(a[:, 0])
        v = _v_of(code, a)
    else:
        s["m"], s["v"] = m.view(-1), v.view(-1)
    if s["param"] is not None:
        s["param"].copy_(s["w"])
    out = {"w": s["w"], "m": m.reshape(-1), "v": v.reshape(-1)}
    return out | ({"param": s["param"]} if s["param"] is not None else {})


# ---- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"embed": _exact_embed, "table": _exact_table, "policy": _exact_policy, "adamw": _exact_adamw}[case["kind"]](s, case)


def _exact_embed(s, c):
    out = torch.zeros(c["T"], c["d"], device="cuda", dtype=torch.float64)
    live = torch.nonzero((s["tokens"] >= 0) & (s["tokens"] < c["V"]))[:, 0]
    out[live] = s["table"].index_select(0, s["tokens"][live].long()).double() * s["scale"]
    return out


def _exact_table(s, c):
    out = s["dTable"].double() if c["add"] else torch.zeros(c["V"], c["d"], device="cuda", dtype=torch.float64)
    live = torch.nonzero((s["tokens"] >= 0) & (s["tokens"] < c["V"]))[:, 0]
    for part in live.split(1 << 14):
        out.index_add_(0, s["tokens"][part].long(), s["dX"][part].double(), alpha=s["scale"])
    return out


def _exact_policy(s, c):
    T, V = c["T"], c["V"]
    inv_tau = float(np.float32(1 / c["tau"]))
    lp = torch.zeros(T, device="cuda", dtype=torch.float64)
    grad = torch.zeros(T, c["ld"], device="cuda", dtype=torch.float64) if c["mode"] == "grad" else None
    sums = torch.zeros(4, device="cuda", dtype=torch.float64)
    step = max(1, (1 << 27) // V)
    for r in range(0, T, step):
        rows = slice(r, min(T, r + step))
        w, A, y = s["weight"][rows].double(), s["advantage"][rows].double(), s["action"][rows].long()[:, None]
        logs = torch.log_softmax(s["logits"][rows, :V].double() * inv_tau, 1)
        mine = logs.gather(1, y)[:, 0]
        lp[rows] = torch.where(w != 0, mine, 0.0)
        if c["mode"] == "logp":
            continue
        ratio = torch.exp(mine - s["old"][rows].double())
        gain = -torch.minimum(ratio * A, ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * A)
        clipped = gain > -ratio * A
        kl = torch.zeros_like(gain)
        slope = torch.where(clipped, 0.0, -ratio * A)
        if c["kl"]:
            near = torch.exp(s["ref"][rows].double() - mine)
            kl = near - (s["ref"][rows].double() - mine) - 1
            slope = slope + KL_COEF * (1 - near)
        sums += torch.stack([((gain + KL_COEF * kl) * w).sum(), (gain * w).sum(), (kl * w).sum(), w[clipped].sum()])
        if grad is not None:
            slope = slope * w * inv_tau
            grad[rows, :V] = -torch.exp(logs) * slope[:, None]
            grad[rows].scatter_add_(1, y, slope[:, None])
    if c["mode"] == "logp":
        return lp
    return {"logp": lp, "stats": sums} | ({"dlogits": grad} if grad is not None else {})


def _exact_adamw(s, c):
    step, blocks = s["step"] + 1, s["decay"].shape[0]
    u_m, u_v = (u.double() for u in _random(dict(s, step=step), blocks)) if c["bits"] == 8 else (None, None)
    g = s["grad"].double().view(blocks, BLOCK) * s["clip"].double()
    if c["bits"] == 8:
        m, v = s["m"].double().view(blocks, BLOCK) / 127, s["v"].double().view(blocks, BLOCK) / 255
        m = m * m.abs() * s["m_scale"].double()[:, None]
        v = v ** 4 * s["v_scale"].double()[:, None]
    else:
        m, v = s["m"].double().view(blocks, BLOCK), s["v"].double().view(blocks, BLOCK)
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g * g
    w = s["w"].double().view(blocks, BLOCK)
    w = w - LR * (m / (1 - BETA1 ** step) / ((v / (1 - BETA2 ** step)).sqrt() + EPS) + s["decay"].double() * DECAY * w)
    if c["bits"] == 8:
        m = _exact_code(m.abs(), 2, 127, u_m) * m.sign()
        v = _exact_code(v, 4, 255, u_v, lowest=1)
    out = {"w": w.view(-1), "m": m.reshape(-1), "v": v.reshape(-1)}
    return out | ({"param": out["w"]} if c["param"] == "bf16" else {})


def _exact_code(x, power, top, u, lowest=0):
    a = x.amax(1, keepdim=True).clamp(min=1e-300)
    part = x / a
    lo = (top * part ** (1 / power)).floor().clamp(0, top - 1)
    below, above = (lo / top) ** power, ((lo + 1) / top) ** power
    code = lo + ((part - below) > u * (above - below)).double()
    return (torch.where(part > 0, code.clamp(min=lowest), 0.0) / top) ** power * a
