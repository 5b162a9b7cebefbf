"""The way into the experts as a whole: a step from rows through norm, gate network, routing by scores and 8-bit experts and back; the argument checks in
C++ and in Python; captured calls; calls on two streams."""
import numpy as np
import pytest
import torch

import harness as Hn
import paper_2504_19925_amd as symi
import workloads as wl
from oracle import way_oracle as O
from paper_2504_19925_amd import binding

pytestmark = pytest.mark.gpu
OTHER = {torch.float32: torch.int32, torch.int32: torch.float32, torch.bfloat16: torch.float16, torch.uint8: torch.int8, torch.float8_e4m3fn: torch.uint8}
U16 = 2.0 ** -8


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(seed, *shape, scale=1.0):
    return torch.randn(*shape, generator=gen(seed), device="cuda") * scale


def codes(ctx, X, groups, rows, n, block):
    q = torch.empty(groups, rows, symi.symi_pitch8(n), dtype=torch.float8_e4m3fn, device="cuda")
    s = torch.empty(groups, -(-rows // block), symi.symi_scale_pitch8(n), dtype=torch.uint8, device="cuda")
    symi.symi_quant8(ctx, X, groups, rows, n, block, q, s)
    return q, s


class Block:
    """One MoE block with a norm in front, as a program would hold it: bf16, classes balanced by a bias."""

    def __init__(self, c, seed=0):
        self.c = c
        self.layer = Hn.State(c)
        self.ctx = self.layer.ctx
        self.layer.place_current()
        T, d, E = c.T, c.d, c.E
        new = lambda *s, dtype=torch.float32: torch.empty(*s, dtype=dtype, device="cuda")   # noqa: E731
        b16 = torch.bfloat16
        self.w, self.b = 1 + randn(seed + 1, d, scale=0.1), randn(seed + 2, d, scale=0.1)
        self.Wr, self.bias = randn(seed + 3, E, d, scale=0.05).to(b16), torch.zeros(E, device="cuda")
        self.hp = symi.SymiScore.make("sigmoid", 4, 2, 2, 1.5)
        self.R, self.N, self.mean, self.rstd = new(T, d, dtype=b16), new(T, d, dtype=b16), new(T), new(T)
        self.logits, self.dlogits, self.dWr = new(T, E), new(T, E), new(E, d)
        self.dR, self.dw, self.db = new(T, d, dtype=b16), new(d), new(d)
        self.nws = new(symi.symi_norm_workspace_bytes(self.ctx), dtype=torch.uint8)
        self.ws8 = new(symi.symi_workspace8_bytes(self.ctx), dtype=torch.uint8)
        L = self.layer
        self.w1, self.w2 = codes(self.ctx, L.W1s, c.S_tot, 2 * c.f, d, 128), codes(self.ctx, L.W2s, c.S_tot, d, c.f, 128)
        # what the products see, for the backward pass
        self.V1, self.V2 = torch.empty_like(L.W1s), torch.empty_like(L.W2s)
        symi.symi_dequant8(self.ctx, *self.w1, c.S_tot, 2 * c.f, d, 128, self.V1)
        symi.symi_dequant8(self.ctx, *self.w2, c.S_tot, d, c.f, 128, self.V2)

    def forward(self, X, residual):
        L, ctx = self.layer, self.ctx
        symi.symi_norm_fwd(ctx, 1, 1e-5, X, residual, self.w, self.b, self.R, self.N, self.mean, self.rstd)
        symi.symi_router_fwd(ctx, self.N, self.Wr, None, self.logits)
        symi.symi_route_scored(ctx, self.hp, self.logits, self.bias, L.idx, L.gate, L.hist)
        symi.symi_dispatch(ctx, self.N, L.idx, L.hist, L.counts, L.first_slot, L.row_of_assign, L.assign_of_row, L.slot_offsets, L.Xp, L.ws)
        symi.symi_expert_fwd8(ctx, L.Xp, L.slot_offsets, *self.w1, *self.w2, L.UV, L.H, L.Yp, self.ws8)
        symi.symi_combine(ctx, L.Yp, L.row_of_assign, L.gate, L.Y)
        return L.Y

    def backward(self, dY):
        """Gradient of X and residual, dY being that of Y, and that of R through the residual stream too."""
        L, ctx = self.layer, self.ctx
        symi.symi_combine_bwd(ctx, dY, L.Yp, L.row_of_assign, L.gate, L.dYp, L.dgate)
        symi.symi_expert_bwd(ctx, L.dYp, L.Xp, L.UV, L.H, L.slot_offsets, L.first_slot, self.V1, self.V2, L.dXp, L.dW1, L.dW2, L.ws)
        symi.symi_dispatch_bwd(ctx, L.dXp, L.row_of_assign, L.dX)
        symi.symi_route_scored_bwd(ctx, self.hp, self.logits, L.idx, L.gate, L.dgate, self.dlogits)
        symi.symi_router_bwd(ctx, self.N, self.Wr, self.dlogits, self.dWr, None, L.dX, L.ws)
        symi.symi_norm_bwd(ctx, 1, L.dX, self.R, self.mean, self.rstd, self.w, dY, self.dR, self.dw, self.db, self.nws)
        symi.symi_route_bias(ctx, L.hist, 1e-3, self.bias)
        return self.dR


def small(**kw):
    return wl.scaled(wl.get_config("c2"), **{**dict(T=160, E=16, k=3, d=136, f=264, S_tot=20, N=1), **kw})


def plain_block(b, X, residual, idx):
    """The block in elementary operations of torch in 64 bits on the CPU, values rounded to 8 bits passing gradients on; classes as chosen."""
    c = b.c
    to64 = lambda t: t.detach().cpu().double()   # noqa: E731
    leaf = lambda t: to64(t).requires_grad_()   # noqa: E731
    R, w, bb, Wr = leaf((X.float() + residual.float()).to(torch.bfloat16)), leaf(b.w), leaf(b.b), leaf(b.Wr)
    mean = R.mean(1, keepdim=True)
    N = (R - mean) / ((R - mean).square().mean(1, keepdim=True) + 1e-5).sqrt() * w + bb
    N = N + (N.detach().float().to(torch.bfloat16).double() - N.detach())      # rounded, gradient 1
    s = torch.sigmoid(N @ Wr.t()).gather(1, idx.cpu().long())
    gate = 1.5 * s / s.sum(1, keepdim=True)

    def eighth(x):
        q, p = O.quant(x.detach().numpy(), 1)
        return x + (torch.from_numpy(O.values(q, p, 1)) - x.detach())

    first = b.layer.first_slot.tolist()
    out = torch.zeros(c.T, c.d, dtype=torch.float64)
    N8 = eighth(N)
    for e in range(c.E):
        t, j = (idx.cpu() == e).nonzero(as_tuple=True)
        if not len(t):
            continue
        uv = N8[t] @ to64(b.V1).view(c.S_tot, 2 * c.f, c.d)[first[e]].t()
        h = torch.nn.functional.silu(uv[:, :c.f]) * uv[:, c.f:]
        y = eighth(h) @ to64(b.V2).view(c.S_tot, c.d, c.f)[first[e]].t()
        out = out.index_add(0, t, gate[t, j][:, None] * y)
    return out, R, w, bb, Wr


def test_a_block_forward_and_back_is_the_formulas():
    """Against binary64 with the same choices.  Outputs are held to a few roundings to bf16 of what they are sums of: 8 stages round activations or their
    gradients to bf16, and those of 8 bits are a part in 2^4 where one falls on the other side of a border (here and there one of hundreds)."""
    c = small()
    b = Block(c)
    X, residual = randn(11, c.T, c.d).to(torch.bfloat16), randn(12, c.T, c.d).to(torch.bfloat16)
    b.bias.copy_(randn(13, c.E, scale=0.02))
    Y = b.forward(X, residual).clone()
    idx = b.layer.idx.clone()
    dY = randn(14, c.T, c.d, scale=0.1).to(torch.bfloat16)
    dR = b.backward(dY)
    want, R, w, bb, Wr = plain_block(b, X, residual, idx)
    (want * dY.cpu().double()).sum().backward()
    far = lambda got, ref: float((got.detach().cpu().double() - ref).norm() / ref.norm())   # noqa: E731
    for name, got, ref in (("Y", Y, want.detach()), ("dR", dR, R.grad + dY.cpu().double()), ("dw", b.dw, w.grad), ("db", b.db, bb.grad), ("dWr", b.dWr, Wr.grad)):
        print(f"[way] {name} {far(got, ref):.2e}", flush=True)
        assert far(got, ref) <= 8 * U16, name
    assert (b.layer.hist.sum() == c.T * c.k) and (b.bias != 0).all()


def test_captured_and_replayed():
    """Forward and backward in a graph, replayed over new inputs with eager work in between: the bits of the eager calls."""
    c = small(T=96)
    b = Block(c)
    X, residual, dY = (torch.empty(c.T, c.d, dtype=torch.bfloat16, device="cuda") for _ in range(3))

    def step():
        b.forward(X, residual)
        b.backward(dY)

    def outputs():
        return [t.clone() for t in (b.R, b.N, b.mean, b.rstd, b.layer.idx, b.layer.gate, b.layer.hist, b.layer.Y, b.dR, b.dw, b.db, b.dlogits, b.bias)]

    def inputs(seed):
        for i, t in enumerate((X, residual, dY)):
            t.copy_(randn(seed + i, c.T, c.d))
        b.bias.copy_(randn(seed + 5, c.E, scale=0.02))

    inputs(0)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (10, 20, 30):
        inputs(seed)
        step()
        want = outputs()
        for t in (b.R, b.N, b.dR, b.dw, b.db, b.dlogits, b.layer.Y):
            t.fill_(3.0)
        b.ws8.fill_(0xA5)
        b.nws.fill_(0xA5)
        inputs(seed)
        torch.cuda.synchronize()
        graph.replay()
        assert all(torch.equal(x, y) for x, y in zip(want, outputs()))


def test_two_streams():
    """Two blocks at once on two streams, each with buffers of its own, give what they give one after the other."""
    c = small(T=700, d=264)
    blocks = [Block(c, seed) for seed in (0, 100)]
    inputs = [[randn(50 + 3 * i + j, c.T, c.d).to(torch.bfloat16) for j in range(3)] for i in range(2)]
    outputs = lambda b: [t.clone() for t in (b.R, b.N, b.layer.idx, b.layer.Y, b.dR, b.dw, b.db, b.dlogits)]   # noqa: E731
    want = []
    for b, (X, residual, dY) in zip(blocks, inputs):
        b.forward(X, residual)
        b.backward(dY)
        want.append(outputs(b))
        b.bias.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for s, b, (X, residual, dY) in zip(streams, blocks, inputs):
            with torch.cuda.stream(s):
                b.forward(X, residual)
                b.backward(dY)
                b.bias.zero_()
    torch.cuda.synchronize()
    for b, w in zip(blocks, want):
        assert all(torch.equal(x, y) for x, y in zip(outputs(b), w))


def test_rows_that_a_capacity_drops():
    """Behind the kept rows of symi_dispatch_capacity nothing is read or written: what lies there may be NaN."""
    c = small(T=200)
    b = Block(c)
    L, ctx = b.layer, b.ctx
    X, residual = randn(1, c.T, c.d).to(torch.bfloat16), randn(2, c.T, c.d).to(torch.bfloat16)
    b.forward(X, residual)
    L.Xp.fill_(float("nan"))
    symi.symi_dispatch_capacity(ctx, 20, b.N, L.idx, L.hist, L.counts, L.first_slot, L.row_of_assign, L.assign_of_row, L.slot_offsets, L.Xp, L.ws)
    kept = int(L.slot_offsets[-1])
    assert 0 < kept < c.T * c.k
    for t in (L.UV, L.H, L.Yp):
        t.fill_(5.0)
    symi.symi_expert_fwd8(ctx, L.Xp, L.slot_offsets, *b.w1, *b.w2, L.UV, L.H, L.Yp, b.ws8)
    for t, width in ((L.UV, 2 * c.f), (L.H, c.f), (L.Yp, c.d)):
        t = t.view(-1, width)
        assert torch.isfinite(t[:kept]).all() and (t[kept:] == 5.0).all()


# ---- argument checks

def arguments(dtype):
    T, E, k, d, f, S = 37, 12, 3, 24, 40, 15
    ctx = symi.symi_create(symi.SymiCfg.make(T, E, k, d, f, S, 1, 0, dtype))
    f32, i32, u8, e4m3 = torch.float32, torch.int32, torch.uint8, torch.float8_e4m3fn
    new = lambda *n, dtype=ctx.torch_dtype: torch.zeros(*n, dtype=dtype, device="cuda")   # noqa: E731
    hp = symi.SymiScore.make("softmax", 4, 2, 2, 1.5)
    A = T * k
    idx = torch.arange(A, device="cuda", dtype=i32) % E
    offs = torch.arange(S + 1, device="cuda", dtype=i32)
    row = lambda: new(T, dtype=f32)   # noqa: E731
    col = lambda: new(d, dtype=f32)   # noqa: E731
    ws8 = lambda: new(symi.symi_workspace8_bytes(ctx), dtype=u8)   # noqa: E731
    calls = {
        "symi_norm_fwd": [1, 1e-5, new(T, d), new(T, d), col(), col(), new(T, d), new(T, d), row(), row()],
        "symi_norm_bwd": [1, new(T, d), new(T, d), row(), row(), col(), new(T, d), new(T, d), col(), col(), new(symi.symi_norm_workspace_bytes(ctx), dtype=u8)],
        "symi_route_scored": [hp, new(T, E, dtype=f32), new(E, dtype=f32), new(A, dtype=i32), new(A, dtype=f32), new(E, dtype=i32)],
        "symi_route_scored_bwd": [hp, new(T, E, dtype=f32), idx, new(A, dtype=f32), new(A, dtype=f32), new(T, E, dtype=f32)],
        "symi_route_bias": [new(E, dtype=i32), 0.5, new(E, dtype=f32)],
        "symi_quant8": [new(3, 130, 136), 3, 130, 136, 128, new(3, 130, 256, dtype=e4m3), new(3, 2, 4, dtype=u8)],
        "symi_dequant8": [new(3, 130, 256, dtype=e4m3), new(3, 130, 4, dtype=u8), 3, 130, 136, 1, new(3, 130, 136)],
        "symi_product8": [new(A, 640, dtype=e4m3), new(A, 8, dtype=u8), offs, new(S, 136, 640, dtype=e4m3), new(S, 2, 8, dtype=u8), 136, 520, new(A, 136), ws8()],
        "symi_expert_fwd8": [new(A, d), offs, new(S, 2 * f, 128, dtype=e4m3), new(S, 1, 4, dtype=u8), new(S, d, 128, dtype=e4m3), new(S, 1, 4, dtype=u8),
                             new(A, 2 * f), new(A, f), new(A, d), ws8()],
    }
    if dtype == "f32":
        del calls["symi_expert_fwd8"]
    return {n: [ctx, *a] for n, a in calls.items()}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_exact_sizes_and_types(dtype):
    calls = arguments(dtype)
    assert set(binding.WAY) == set(binding._marshal_way) and set(binding.WAY) - set(calls) <= {"symi_expert_fwd8"}
    for name, args in calls.items():
        fast, call = binding._marshal_way[name], getattr(symi, name)
        assert fast(*args) == 0, name
        call.through_ctypes(*args)
        for i, t in enumerate(args):
            if not isinstance(t, torch.Tensor):
                continue
            for bad in (t.view(-1)[:-1], t.view(OTHER[t.dtype])):
                wrong = args[:i] + [bad] + args[i + 1:]
                assert fast(*wrong) is None, (name, i)
                said = []
                for f in (call, call.through_ctypes):
                    with pytest.raises(symi.SymiError, match="needs at least|expected dtype") as e:
                        f(*wrong)
                    said.append(str(e.value))
                assert said[0] == said[1], name
        assert fast(*args[:-1]) is None
        with pytest.raises(TypeError):
            call(*args[:-1])
    torch.cuda.synchronize()


def test_what_may_be_left_out_and_numbers_of_other_kinds():
    calls = arguments("bf16")
    for name, gone in (("symi_norm_fwd", (4, 7)), ("symi_norm_fwd", (5, 6)), ("symi_norm_fwd", (9, 10)), ("symi_norm_bwd", (6, 7)), ("symi_norm_bwd", (9,)),
                       ("symi_norm_bwd", (10,)), ("symi_route_scored", (3,)), ("symi_expert_fwd8", (7, 8))):
        args = [None if i in gone else x for i, x in enumerate(calls[name])]
        assert binding._marshal_way[name](*args) == 0
        getattr(symi, name).through_ctypes(*args)
    args = list(calls["symi_route_bias"])
    args[2] = 1                                       # not the plain type: the Python path takes it
    assert binding._marshal_way["symi_route_bias"](*args) is None
    symi.symi_route_bias(*args)
    args = list(calls["symi_quant8"])
    args[2] = np.int64(3)
    assert binding._marshal_way["symi_quant8"](*args) is None
    symi.symi_quant8(*args)
    symi.symi_quant8(args[0], X=args[1], groups=3, rows=130, n=136, block=128, q=args[6], s=args[7])
    for i, bad in ((2, -1), (3, 2 ** 31 - 1), (5, 0)):
        args = list(calls["symi_quant8"])
        args[i] = bad
        assert binding._marshal_way["symi_quant8"](*args) is None
        with pytest.raises(symi.SymiError):
            symi.symi_quant8(*args)
    torch.cuda.synchronize()


def test_a_timing_context_books_every_kernel():
    c = small(T=3000)
    ctx = Hn.make_ctx(c, flags=symi.CTX_TIMING)
    b = Block(c)
    L = b.layer
    b.forward(randn(1, c.T, c.d).to(torch.bfloat16), randn(2, c.T, c.d).to(torch.bfloat16))
    x, q, s = b.N, torch.empty(c.T, 256, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(c.T, 4, dtype=torch.uint8, device="cuda")
    for call, kernels in (
            (lambda: symi.symi_norm_fwd(ctx, 1, 1e-5, x, None, b.w, b.b, None, b.R, b.mean, b.rstd), {"norm"}),
            (lambda: symi.symi_norm_bwd(ctx, 1, x, b.R, b.mean, b.rstd, b.w, None, b.dR, b.dw, b.db, b.nws), {"norm_bwd", "norm_sum"}),
            (lambda: symi.symi_route_scored(ctx, b.hp, b.logits, b.bias, L.idx, L.gate, L.hist), {"route_scored"}),
            (lambda: symi.symi_route_scored_bwd(ctx, b.hp, b.logits, L.idx, L.gate, L.dgate, b.dlogits), {"route_scored_bwd"}),
            (lambda: symi.symi_route_bias(ctx, L.hist, 0.1, b.bias), {"route_bias"}),
            (lambda: symi.symi_quant8(ctx, x, 1, c.T, c.d, 1, q, s), {"quant8"}),
            (lambda: symi.symi_dequant8(ctx, q, s, 1, c.T, c.d, 1, x), {"dequant8"}),
            (lambda: symi.symi_expert_fwd8(ctx, L.Xp, L.slot_offsets, *b.w1, *b.w2, L.UV, L.H, L.Yp, b.ws8), {"quant8", "expert8", "product8"})):
        symi.symi_timing_reset(ctx)
        call()
        torch.cuda.synchronize()
        seen = {symi.symi_kernel_name(i): symi.symi_timing_read(ctx, i) for i in range(symi.symi_kernel_count())}
        assert kernels <= {name for name, (_, n) in seen.items() if n} <= kernels | {"fill_i32", "tiles8"}
        assert all(ms > 0 for ms, n in seen.values() if n)
