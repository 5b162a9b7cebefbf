"""AdamW over many tensors against binary64: every kind of tensor, ragged sizes, 8-bit states and what they do over many steps.

Bounds (u = 2^-24).  m: three roundings of its two summands; v: four.  The weight: its update is a quotient of m and the root
of v, each with a handful of roundings (16 u together), and inherits m's and half of v's relative error; the subtraction
rounds once more.  An 8-bit code is the oracle's wherever the choice between its two neighbours is not within 1e-4 of the
random number or of a code (fp32 values are off by 4 u of steps that are 1/100 of them: 3e-5), and one off at most elsewhere."""
import ctypes

import numpy as np
import pytest
import torch

import harness as Hn
import paper_2504_19925_amd as symi
from oracle import ends_oracle as O

pytestmark = pytest.mark.gpu
U32, U16 = 2.0 ** -24, 2.0 ** -8
HP = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-6, wd=0.1)
HP = {k: float(np.float32(v)) for k, v in HP.items()}


def context(flags=0):
    return symi.symi_create(symi.SymiCfg.make(1, 1, 1, 8, 8, 1, 1, 0, "f32"), flags)


def adam(step, gscale=1.0, **kw):
    h = {**HP, **kw}
    return symi.SymiAdam(h["lr"], h["beta1"], h["beta2"], h["eps"], h["wd"], gscale, step)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def shifted(t, by):
    flat = torch.empty(t.numel() + by, dtype=t.dtype, device="cuda")
    flat[by:] = t.reshape(-1)
    return flat[by:].view(t.shape)


def make(n, param="f32", grad="f32", bits=32, decay=1.0, seed=0, by=0, fresh=False):
    """One tensor in the middle of its training (or at its start: `fresh`)."""
    g = gen(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    nb = -(-n // 256)
    w = randn(n) * 0.05
    t = {"grad": (randn(n) * torch.exp(randn(n))).to(torch.bfloat16 if grad == "bf16" else torch.float32), "decay": decay}
    if param == "bf16":
        t["master"], t["param"] = w, w.to(torch.bfloat16)
    else:
        t["param"] = w
    if bits == 8:
        t["m"] = torch.randint(-127, 128, (n,), generator=g, device="cuda", dtype=torch.int8)
        t["v"] = torch.randint(0, 256, (n,), generator=g, device="cuda", dtype=torch.int16).to(torch.uint8)
        t["m_scale"], t["v_scale"] = torch.exp(randn(nb)) * 0.1, torch.exp(randn(nb)) * 0.1
    else:
        t["m"], t["v"] = randn(n) * 0.3, randn(n).square() * 0.1
    if fresh:
        for k in ("m", "v", "m_scale", "v_scale"):
            if k in t:
                t[k].zero_()
    return {k: shifted(x, by) if isinstance(x, torch.Tensor) and by else x for k, x in t.items()}


def states(t):
    """(m, v) in binary64."""
    if t["m"].dtype == torch.int8:
        return O.m_values(Hn.npf(t["m"]), Hn.npf(t["m_scale"])), O.v_values(Hn.npf(t["v"]), Hn.npf(t["v_scale"]))
    return Hn.npf(t["m"]).astype(np.float64), Hn.npf(t["v"]).astype(np.float64)


def snapshot(tensors):
    return [{k: x.clone() if isinstance(x, torch.Tensor) else x for k, x in t.items()} for t in tensors]


def check(before, after, step, gscale=1.0, seed=0):
    """`after` is `before` a step on."""
    first = 0
    for i, (b, a) in enumerate(zip(before, after)):
        n = b["param"].numel()
        if n == 0:
            continue
        w0 = Hn.npf(b.get("master", b["param"])).astype(np.float64)
        g = Hn.npf(b["grad"]).astype(np.float64)
        m0, v0 = states(b)
        w, m, v = O.adamw(w0, g, m0, v0, HP["lr"], HP["beta1"], HP["beta2"], HP["eps"], HP["wd"] * b["decay"], step, gscale)
        dm = 4 * U32 * (np.abs(HP["beta1"] * m0) + np.abs((1 - HP["beta1"]) * gscale * g)) + 1e-45
        dv = 6 * U32 * v + 1e-45
        root = np.sqrt(v / (1 - HP["beta2"] ** step)) + HP["eps"]
        up = np.abs(m) / (1 - HP["beta1"] ** step) / root
        tol = 2 * U32 * (np.abs(w0) + np.abs(w)) + HP["lr"] * (dm / (1 - HP["beta1"] ** step) / root + 20 * U32 * up + 4 * U32 * HP["wd"] * np.abs(w0))
        assert (np.abs(Hn.npf(a.get("master", a["param"])) - w) <= tol).all(), i
        if "master" in b and b["master"] is not None:
            assert torch.equal(a["param"], a["master"].to(torch.bfloat16)), i
        if b["m"].dtype == torch.int8:
            um, uv = O.random_numbers(seed, step, first, n)
            for name, x, power, top, u, scale in (("m", np.abs(m), 2, 127, um, "m_scale"), ("v", v, 4, 255, uv, "v_scale")):
                big = O.block_max(x)
                assert (np.abs(Hn.npf(a[scale]) - big) <= 1e-5 * big).all(), (i, name)
                code, near = O.encode(x, power, top, u)
                got = Hn.npf(a[name]).astype(np.int64)
                if name == "m":
                    assert (np.sign(got) * np.sign(m) >= 0).all(), i
                    got = np.abs(got)
                else:
                    code = np.where(x > 0, np.maximum(code, 1), 0)
                off = np.abs(got - code)
                assert (off <= (near < 1e-4)).all(), (i, name, off.max(), int((off > (near < 1e-4)).sum()))
        else:
            assert (np.abs(Hn.npf(a["m"]) - m) <= dm).all() and (np.abs(Hn.npf(a["v"]) - v) <= dv).all(), i
        first += -(-n // 256)


SIZES = [1, 3, 4, 255, 256, 257, 1023, 4095, 4096, 4097, 16384, 50001, 0, 2]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("param", ["f32", "bf16"])
def test_steps(param, grad, bits):
    ctx = context()
    tensors = [make(n, param, grad, bits, (1.0, 0.0, 0.5)[i % 3], i) for i, n in enumerate(SIZES)]
    opt = symi.symi_adamw_create(tensors)
    assert symi.symi_adamw_values(opt) == sum(-(-n // 256) * 256 for n in SIZES)
    for step, scale, seed in ((7, None, 1), (8, 0.25, 2), (9, -3.0, 2 ** 32 - 1)):
        before = snapshot(tensors)
        clip = None if scale is None else torch.full((1,), scale, device="cuda")
        symi.symi_adamw_step(ctx, opt, adam(step, 0.5), clip, seed)
        check(before, tensors, step, 0.5 * (1.0 if scale is None else scale), seed)


def test_every_kind_in_one_call_at_any_alignment():
    ctx = context()
    kinds = [(p, g, b) for p in ("f32", "bf16") for g in ("f32", "bf16") for b in (8, 32)]
    tensors = [make(n, *kinds[i % 8], decay=float(i % 2), seed=i, by=1 + i % 3) for i, n in enumerate((70, 9000, 513, 4096, 1, 3333, 256, 8, 700) * 3)]
    opt = symi.symi_adamw_create(tensors)
    before = snapshot(tensors)
    symi.symi_adamw_step(ctx, opt, adam(3), None, 5)
    check(before, tensors, 3, 1.0, 5)
    # the decoded states, and nothing between them
    n = symi.symi_adamw_values(opt)
    m, v = torch.full((n,), -7.0, device="cuda"), torch.full((n,), -7.0, device="cuda")
    symi.symi_adamw_decode(ctx, opt, m, v)
    at = 0
    for t in tensors:
        size = t["param"].numel()
        m64, v64 = states(t)
        assert (np.abs(Hn.npf(m[at:at + size]) - m64) <= 4 * U32 * np.abs(m64)).all()
        assert (np.abs(Hn.npf(v[at:at + size]) - v64) <= 6 * U32 * v64).all()
        end = at + -(-size // 256) * 256
        assert (m[at + size:end] == -7).all() and (v[at + size:end] == -7).all()
        at = end


def test_nothing_beside_the_tensors_is_written():
    """Tensors inside larger buffers: what lies before and behind them stays."""
    ctx = context()
    for n in (1, 5, 255, 4099):
        whole = make(n + 32, "bf16", "f32", 8, seed=n)
        t = {k: (x[16:16 + n] if x.numel() == n + 32 else x[:-(-n // 256)]) if isinstance(x, torch.Tensor) else x for k, x in whole.items()}
        scales = {k: torch.cat([whole[k][:-(-n // 256)], torch.full((4,), 5.0, device="cuda")]) for k in ("m_scale", "v_scale")}
        t.update({k: x[:-4] for k, x in scales.items()})
        before = snapshot([whole])[0]
        opt = symi.symi_adamw_create([t])
        symi.symi_adamw_step(ctx, opt, adam(1), None, 0)
        for k in ("param", "master", "m", "v"):
            assert torch.equal(whole[k][:16], before[k][:16]) and torch.equal(whole[k][16 + n:], before[k][16 + n:]), k
            assert not torch.equal(whole[k], before[k]) or n < 8
        assert all((x[-4:] == 5).all() for x in scales.values())


def test_a_fresh_state_and_blocks_without_gradient():
    ctx = context()
    tensors = [make(2000, "f32", "f32", bits, seed=9, fresh=True) for bits in (32, 8)]
    for t in tensors:
        t["grad"][256:768] = 0           # rows that no token chose
        t["grad"][1000] = 0
    before = snapshot(tensors)
    opt = symi.symi_adamw_create(tensors)
    symi.symi_adamw_step(ctx, opt, adam(1), None, 0)
    check(before, tensors, 1)
    t = tensors[1]
    assert not t["m"][256:768].any() and not t["v"][256:768].any() and not t["v_scale"][1:3].any()
    assert t["v"][1000] == 0 and (t["v"][:256] > 0).all()     # a value above 0 never becomes 0
    assert (t["param"] - tensors[0]["param"]).abs().max() <= 1e-7   # the first update is that of the exact states


def test_the_mean_of_what_is_stored_is_the_value():
    """The same step with 4096 seeds: the mean of a stored value is within 6 standard errors of the exact one; so are the ones
    that the nearest code would never reach."""
    ctx = context()
    n, seeds = 256, 4096
    base = make(n, bits=8, seed=3)
    base["grad"] *= 1e-3                  # v decays, by 1 % here
    want_m, want_v = O.adamw(Hn.npf(base["param"]), Hn.npf(base["grad"]), *states(base), HP["lr"], HP["beta1"], HP["beta2"], HP["eps"], 0.0, 5)[1:]
    many = {k: torch.cat([x] * seeds) if isinstance(x, torch.Tensor) else x for k, x in base.items()}   # every block has random numbers of its own
    opt = symi.symi_adamw_create([many])
    symi.symi_adamw_step(ctx, opt, adam(5), None, 77)
    m, v = (torch.empty(n * seeds, device="cuda") for _ in range(2))
    symi.symi_adamw_decode(ctx, opt, m, v)
    for got, want, floor in ((m, want_m, 0.0), (v, want_v, want_v.max() / 255 ** 4)):
        x = Hn.npf(got).astype(np.float64).reshape(seeds, n)
        error = 6 * x.std(axis=0) / np.sqrt(seeds) + 1e-5 * np.abs(want)
        # a probability is taken in steps of 2^-16, and v below code 1 is code 1
        step = np.maximum(np.abs(want), floor) * 0.2
        assert (np.abs(x.mean(axis=0) - want) <= error + step * 2.0 ** -16 + floor).all()
    assert (Hn.npf(v).reshape(seeds, n).std(axis=0) > 0).mean() > 0.5


def test_8_bit_states_follow_32_bit_ones():
    """300 steps of a noisy quadratic, then gradients that are a tenth: v has to come down by its own decay.  Its mean over the
    tensor follows the 32-bit one to 3 %, and the weights end as near to the minimum."""
    ctx = context()
    n = 256 * 64
    w0 = torch.randn(n, generator=gen(1), device="cuda")
    opts, ts = [], []
    for bits in (32, 8):
        t = make(n, bits=bits, seed=0, fresh=True, decay=0.0)
        t["param"].copy_(w0)
        ts.append(t)
        opts.append(symi.symi_adamw_create([t]))
    g = gen(2)
    for step in range(1, 601):
        noise = torch.randn(n, generator=g, device="cuda")
        for t, o in zip(ts, opts):
            t["grad"].copy_((t["param"] + 0.5 * noise) * (1.0 if step <= 300 else 0.1))
            symi.symi_adamw_step(ctx, o, adam(step, lr=0.01), None, 11)
    m, v = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    symi.symi_adamw_decode(ctx, opts[1], m, v)
    assert abs(v.mean() / ts[0]["v"].mean() - 1) < 0.03
    a, b = (t["param"].square().mean().item() for t in ts)
    assert b < 1.2 * a + 1e-3 and (ts[0]["param"] - ts[1]["param"]).square().mean() < 0.2 * max(a, 1e-3) + 0.01


def test_values_that_are_not_finite():
    ctx = context()
    for bits in (32, 8):
        t = make(1024, bits=bits, seed=4)
        clean = snapshot([t])[0]
        t["grad"][300], t["grad"][600] = float("nan"), float("inf")
        before = snapshot([t])
        opts = [symi.symi_adamw_create([x]) for x in (t, clean)]
        for o in opts:
            symi.symi_adamw_step(ctx, o, adam(2), None, 0)
        hit = torch.zeros(1024, dtype=torch.bool, device="cuda")
        hit[[300, 600]] = True
        assert t["param"][300].isnan() and t["param"][600].isnan()
        assert torch.equal(t["param"][~hit], clean["param"][~hit])       # no other weight
        if bits == 8:      # a scale stands for 256 values: those blocks are lost, loudly, and no others
            assert t["m_scale"][1].isnan() and t["v_scale"][2].isnan() and not t["m"][256:768].any()
            assert torch.equal(t["m"][768:], clean["m"][768:]) and torch.equal(t["m_scale"][[0, 3]], clean["m_scale"][[0, 3]])
            m, v = torch.empty(1024, device="cuda"), torch.empty(1024, device="cuda")
            symi.symi_adamw_decode(ctx, opts[0], m, v)
            assert m[256:768].isnan().all() and not m[:256].isnan().any()
        del before


def test_tiny_and_huge_values():
    """Gradients of 1e-22 (v is a denormal number: stored as zeros, the weight does not move beyond the rate) and of 1e18."""
    ctx = context()
    for scale in (1e-22, 1e-30, 1e18):
        tensors = [make(600, bits=bits, seed=6, fresh=True) for bits in (32, 8)]
        for t in tensors:
            t["grad"] *= scale
        opts = [symi.symi_adamw_create([t]) for t in tensors]
        before = snapshot(tensors)
        for step in (1, 2, 3):
            for o in opts:
                symi.symi_adamw_step(ctx, o, adam(step), None, 0)
        for t, b in zip(tensors, before):
            assert t["param"].isfinite().all()
            assert ((t["param"] - b["param"]).abs() <= 3 * HP["lr"] * (3.0 + HP["wd"] * b["param"].abs())).all()


def test_offsets_beyond_32_bits():
    """One tensor of more than 2^31 values, 8-bit states: its last values, and some in the middle, as a tensor of their own."""
    ctx = context()
    n = 2 ** 31 + 3 * 256 + 77
    t = {"param": torch.zeros(n, device="cuda"), "grad": torch.zeros(n, device="cuda", dtype=torch.bfloat16), "decay": 1.0,
         "m": torch.zeros(n, device="cuda", dtype=torch.int8), "v": torch.zeros(n, device="cuda", dtype=torch.uint8),
         "m_scale": torch.zeros(-(-n // 256), device="cuda"), "v_scale": torch.zeros(-(-n // 256), device="cuda")}
    spots = [(0, 256), (2 ** 30, 512), (2 ** 31 - 256, 512), (n - 77 - 256, 256 + 77)]
    for at, size in spots:
        part = make(size, "f32", "bf16", 8, seed=size)
        for k in ("param", "grad", "m", "v"):
            t[k][at:at + size] = part[k]
        for k in ("m_scale", "v_scale"):
            t[k][at // 256:-(-(at + size) // 256)] = part[k]
    cut = lambda at, size: {k: (x[at // 256:-(-(at + size) // 256)] if "scale" in k else x[at:at + size]).clone() if k != "decay" else x   # noqa: E731
                            for k, x in t.items()}
    before = [cut(*s) for s in spots]
    opt = symi.symi_adamw_create([t])
    symi.symi_adamw_step(ctx, opt, adam(4), None, 9)
    for (at, size), b in zip(spots, before):
        a = cut(at, size)
        w, m, v = O.adamw(Hn.npf(b["param"]), Hn.npf(b["grad"]), *states(b), HP["lr"], HP["beta1"], HP["beta2"], HP["eps"], HP["wd"], 4)
        assert np.abs(Hn.npf(a["param"]) - w).max() <= 1e-5
        code, near = O.encode(np.abs(m), 2, 127, O.random_numbers(9, 4, at // 256, size)[0])
        assert (np.abs(np.abs(Hn.npf(a["m"]).astype(np.int64)) - code) <= (near < 1e-4)).all()
    for at, size in spots:
        t["m"][at:at + size] = 0
        t["param"][at:at + size] = 0
    assert not t["m"].any() and not t["param"].any()


def test_another_stream_and_a_graph():
    """A step captured into a graph: hp is read when the call is recorded, the clip factor when it runs."""
    ctx = context()
    tensors = [make(n, "bf16", "f32", 8, seed=n) for n in (5000, 300)]
    opt = symi.symi_adamw_create(tensors)
    start = snapshot(tensors)
    clip = torch.ones(1, device="cuda")

    def restore():
        for t, s in zip(tensors, start):
            for k, x in t.items():
                if isinstance(x, torch.Tensor):
                    x.copy_(s[k])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        symi.symi_adamw_step(ctx, opt, adam(6), clip, 3)
    side.synchronize()
    check(start, tensors, 6, 1.0, 3)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        symi.symi_adamw_step(ctx, opt, adam(6), clip, 3)
    for factor in (0.5, 2.0, 0.125):
        restore()
        clip.fill_(factor)
        graph.replay()
        torch.cuda.synchronize()
        check(start, tensors, 6, factor, 3)


def test_refusals():
    ctx = context()
    t = make(300, "bf16", "f32", 8)
    for change in (dict(master=None), dict(m_scale=None), dict(v_scale=None), dict(m=t["m"].to(torch.uint8)), dict(v=t["v"].to(torch.int8)),
                   dict(grad=t["grad"][:-1]), dict(grad=t["grad"].double()), dict(param=t["param"].to(torch.float16)), dict(m=t["m"][:-1]),
                   dict(m_scale=t["m_scale"][:-1]), dict(master=t["master"].cpu()), dict(decay=-1.0), dict(decay=float("nan")),
                   dict(rate=1.0), dict(m=None), dict(param=t["param"].float())):
        with pytest.raises(symi.SymiError):
            symi.symi_adamw_create([t, {**t, **change}])
    opt = symi.symi_adamw_create([t])
    for kw in (dict(beta1=1.0), dict(beta2=-0.1), dict(eps=0.0), dict(eps=float("nan")), dict(beta1=float("nan"))):
        with pytest.raises(symi.SymiError):
            symi.symi_adamw_step(ctx, opt, adam(1, **kw), None, 0)
    with pytest.raises(symi.SymiError, match="step"):
        symi.symi_adamw_step(ctx, opt, adam(0), None, 0)
    with pytest.raises(symi.SymiError):
        symi.symi_adamw_step(ctx, opt, adam(1), torch.ones(1), 0)
    with pytest.raises(symi.SymiError):
        symi.symi_adamw_decode(ctx, opt, torch.empty(511, device="cuda"), torch.empty(512, device="cuda"))
    L = symi.lib()
    assert L.symi_adamw_step(ctx.ptr, None, ctypes.byref(adam(1)), None, 0, None) == -1
    assert L.symi_adamw_step(None, opt.ptr, ctypes.byref(adam(1)), None, 0, None) == -1
    symi.symi_adamw_destroy(opt)
    symi.symi_adamw_destroy(opt)                 # a second destroy of the handle is a no-op
    empty = symi.symi_adamw_create([])
    symi.symi_adamw_step(ctx, empty, adam(1), None, 0)
    assert symi.symi_adamw_values(empty) == 0
