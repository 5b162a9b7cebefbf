"""Token embedding and its gradient against binary64, at the sizes and tokens where they can go wrong.

Bounds: an output of the lookup is one fp32 product, rounded once more in bf16.  A row of the gradient is an fp32 sum of n
terms in some order, times the scale, plus the old value: at most n + 2 roundings of partial sums that no summand exceeds."""
import numpy as np
import pytest
import torch

import harness as Hn
import paper_2504_19925_amd as symi
from oracle import ends_oracle as O

pytestmark = pytest.mark.gpu
U32, U16 = 2.0 ** -24, 2.0 ** -8     # half a unit in the last place is at most this part of an fp32 / a bf16 value


def context(T, d, dtype, flags=0):
    return symi.symi_create(symi.SymiCfg.make(T, 1, 1, d, 8, 1, 1, 0, dtype), flags)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def make_tokens(kind, T, V, seed=0):
    g = gen(seed)
    t = torch.randint(0, V, (T,), generator=g, device="cuda")
    if kind == "skewed":       # a few rows get most tokens
        t = (t.double() / V).pow(6).mul(V).long()
    elif kind == "same":
        t = torch.full_like(t, V - 1)
    elif kind == "padded":     # tokens on both sides of the table
        t = torch.where(torch.rand(T, generator=g, device="cuda") < 0.4, -1 - t, t)
        t[::7] = V
        t[::11] = 2 ** 31 - 1
        t[::13] = -2 ** 31
    elif kind == "none":
        t = torch.full_like(t, -1)
    elif kind == "few":        # three rows of a large table
        t = t % 3 * (V // 3)
    return t.to(torch.int32)


def shifted(t, by):
    """The same values, `by` elements behind an aligned address."""
    flat = torch.empty(t.numel() + by, dtype=t.dtype, device="cuda")
    flat[by:] = t.reshape(-1)
    return flat[by:].view(t.shape)


def backward(ctx, tokens, dX, V, scale, old=None, ws=None):
    dTable = torch.full((V, ctx.d), float("nan"), device="cuda") if old is None else old.clone()
    ws = torch.full((symi.symi_embed_workspace_bytes(ctx, V),), 0xA5, dtype=torch.uint8, device="cuda") if ws is None else ws
    symi.symi_embed_bwd(ctx, tokens, dX, V, scale, int(old is not None), dTable, ws)
    return dTable


def check_gradient(tokens, dX, V, scale, got, old=None):
    want, size, count = O.embed_gradient(tokens.cpu().numpy(), Hn.npf(dX), V, scale)
    if old is not None:
        o = Hn.npf(old)
        rows = count > 0
        assert (Hn.npf(got)[~rows] == o[~rows]).all()      # not touched
        want, size = want + o, size + np.abs(o)
    assert (np.abs(Hn.npf(got) - want) <= (count + 2)[:, None] * U32 * size).all()


SIZES = [(1, 8, 1), (1, 128, 1000), (2, 8, 3), (63, 16, 300), (64, 264, 64), (65, 520, 1025), (257, 128, 8000), (1024, 128, 8000),
         (1023, 1032, 77), (3001, 64, 5003), (4099, 40, 300), (9001, 8, 20011), (20000, 24, 70001)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,V", SIZES)
def test_lookup_and_gradient(T, d, V, dtype):
    ctx = context(T, d, dtype)
    dt = ctx.torch_dtype
    for i, kind in enumerate(("uniform", "skewed", "padded", "same", "none", "few")):
        print(f"[embed] {dtype} T={T} d={d} V={V} {kind}", flush=True)
        scale = (1.0, 0.37, -2.5)[i % 3]
        tokens = make_tokens(kind, T, V, i)
        table = torch.randn(V, d, generator=gen(i), device="cuda").to(dt)
        X = torch.full((T, d), float("nan"), device="cuda", dtype=dt)
        symi.symi_embed_fwd(ctx, tokens, table, V, scale, X)
        want = O.embed(tokens.cpu().numpy(), Hn.npf(table), np.float32(scale).astype(np.float64))
        err = np.abs(Hn.npf(X) - want)
        assert (err <= (U32 + (U16 if dtype == "bf16" else 0)) * 1.01 * np.abs(want)).all()
        dX = torch.randn(T, d, generator=gen(100 + i), device="cuda").to(dt)
        scale64 = float(np.float32(scale))
        check_gradient(tokens, dX, V, scale64, backward(ctx, tokens, dX, V, scale))
        old = torch.randn(V, d, generator=gen(200 + i), device="cuda")
        check_gradient(tokens, dX, V, scale64, backward(ctx, tokens, dX, V, scale, old), old)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_any_alignment_and_the_same_bits_again(dtype):
    T, d, V = 700, 136, 401
    ctx = context(T, d, dtype)
    tokens = make_tokens("skewed", T, V, 3)
    table = torch.randn(V, d, generator=gen(1), device="cuda").to(ctx.torch_dtype)
    dX = torch.randn(T, d, generator=gen(2), device="cuda").to(ctx.torch_dtype)
    X = torch.empty(T, d, device="cuda", dtype=ctx.torch_dtype)
    symi.symi_embed_fwd(ctx, tokens, table, V, 0.5, X)
    dT = backward(ctx, tokens, dX, V, 0.5)
    for by in (1, 3):
        X2 = shifted(torch.zeros_like(X), by)
        symi.symi_embed_fwd(ctx, shifted(tokens, by), shifted(table, by), V, 0.5, X2)
        assert torch.equal(X, X2)
        d2 = shifted(torch.full_like(dT, float("nan")), by)
        ws = torch.empty(symi.symi_embed_workspace_bytes(ctx, V) + 64, dtype=torch.uint8, device="cuda")[by:]
        symi.symi_embed_bwd(ctx, shifted(tokens, by), shifted(dX, by), V, 0.5, 0, d2, ws)
        assert torch.equal(dT, d2)


def test_values_that_are_no_numbers_stay_in_their_rows():
    T, d, V = 300, 64, 50
    ctx = context(T, d, "bf16")
    tokens = make_tokens("uniform", T, V, 4)
    table = torch.randn(V, d, generator=gen(5), device="cuda").to(torch.bfloat16)
    table[7, 3], table[9] = float("nan"), float("inf")
    X = torch.empty(T, d, device="cuda", dtype=torch.bfloat16)
    symi.symi_embed_fwd(ctx, tokens, table, V, 2.0, X)
    assert torch.equal(X.isnan(), table.isnan()[tokens.long()]) and torch.equal(X.isinf(), table.isinf()[tokens.long()])
    dX = torch.randn(T, d, generator=gen(6), device="cuda").to(torch.bfloat16)
    dX[11, 5] = float("nan")
    tokens[12] = -1
    dX[12] = float("nan")                     # padding: not read into any row
    dT = backward(ctx, tokens, dX, V, 1.0)
    bad = torch.zeros_like(dT, dtype=torch.bool)
    bad[tokens[11].long(), 5] = True
    assert torch.equal(dT.isnan(), bad)


def test_gradient_is_that_of_the_lookup():
    """<dX, X(table + D) - X(table)> = <dTable, D>: the lookup is linear, so one difference is exact up to rounding."""
    T, d, V = 500, 72, 90
    ctx = context(T, d, "f32")
    tokens = make_tokens("padded", T, V, 5)
    table, D = (torch.randn(V, d, generator=gen(s), device="cuda") for s in (1, 2))
    dX = torch.randn(T, d, generator=gen(3), device="cuda")
    X = [torch.empty(T, d, device="cuda") for _ in range(2)]
    symi.symi_embed_fwd(ctx, tokens, table, V, 1.5, X[0])
    symi.symi_embed_fwd(ctx, tokens, table + D, V, 1.5, X[1])
    dT = backward(ctx, tokens, dX, V, 1.5)
    a, b = (dX.double() * (X[1].double() - X[0].double())).sum(), (dT.double() * D.double()).sum()
    # table + D, the two lookups and the sums of dT (of at most `most` terms, and two roundings more) are rounded
    size = (dX.double().abs() * (X[1].double().abs() + X[0].double().abs())).sum()
    most = int(torch.bincount(tokens[(tokens >= 0) & (tokens < V)]).max())
    assert abs(a - b) <= (most + 4) * U32 * size


def test_offsets_beyond_32_bits():
    """A table of more than 2^32 bytes and 2^31 elements."""
    T, d, V = 5, 4096, 530000
    ctx = context(T, d, "bf16")
    tokens = torch.tensor([V - 1, 0, V - 2, V - 1, 524289], dtype=torch.int32, device="cuda")
    table = torch.zeros(V, d, dtype=torch.bfloat16, device="cuda")
    live = tokens.long().unique()
    table[live] = torch.randn(len(live), d, generator=gen(1), device="cuda").to(torch.bfloat16)
    X = torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
    symi.symi_embed_fwd(ctx, tokens, table, V, 1.0, X)
    assert torch.equal(X, table[tokens.long()])
    del table
    dX = torch.randn(T, d, generator=gen(2), device="cuda").to(torch.bfloat16)
    dT = backward(ctx, tokens, dX, V, 1.0)
    assert torch.equal(dT[0], dX[1].float()) and torch.equal(dT[V - 2], dX[2].float()) and torch.equal(dT[524289], dX[4].float())
    assert torch.equal(dT[V - 1], dX[0].float() + dX[3].float())
    dT[live] = 0
    assert not dT.any()


def test_no_tokens():
    ctx = context(0, 16, "f32")
    empty = torch.empty(0, dtype=torch.int32, device="cuda")
    rows = torch.empty(0, 16, device="cuda")
    symi.symi_embed_fwd(ctx, empty, torch.ones(9, 16, device="cuda"), 9, 1.0, rows)
    assert not backward(ctx, empty, rows, 9, 1.0).any()
    old = torch.randn(9, 16, device="cuda")
    assert torch.equal(backward(ctx, empty, rows, 9, 1.0, old), old)


def test_another_stream_and_a_graph():
    """Calls on a side stream, then captured and replayed on new inputs, with work of the program's own in between."""
    T, d, V = 2500, 128, 997
    ctx = context(T, d, "bf16")
    side = torch.cuda.Stream()
    dX = torch.randn(T, d, generator=gen(1), device="cuda").to(torch.bfloat16)
    tokens = make_tokens("skewed", T, V, 1)
    dT, ws = torch.empty(V, d, device="cuda"), torch.empty(symi.symi_embed_workspace_bytes(ctx, V), dtype=torch.uint8, device="cuda")
    want = backward(ctx, tokens, dX, V, 1.0)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        symi.symi_embed_bwd(ctx, tokens, dX, V, 1.0, 0, dT, ws)
    side.synchronize()
    assert torch.equal(dT, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        symi.symi_embed_bwd(ctx, tokens, dX, V, 1.0, 0, dT, ws)
    for i in range(4):
        tokens.copy_(make_tokens(("uniform", "same", "padded", "few")[i], T, V, 10 + i))
        want = backward(ctx, tokens, dX, V, 1.0)
        dT.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dT, want)


def test_refusals():
    T, d, V = 8, 16, 9
    ctx = context(T, d, "bf16")
    tokens, ws = torch.zeros(T, dtype=torch.int32, device="cuda"), torch.empty(symi.symi_embed_workspace_bytes(ctx, V), dtype=torch.uint8, device="cuda")
    table, X = torch.zeros(V, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, d, dtype=torch.bfloat16, device="cuda")
    dT = torch.zeros(V, d, device="cuda")
    for bad in ((tokens.long(), table, V, 1.0, X), (tokens, table.float(), V, 1.0, X), (tokens, table, V + 1, 1.0, X),
                (tokens[:-1], table, V, 1.0, X), (tokens, table, V, 1.0, X[:-1]), (tokens, table, 0, 1.0, X),
                (tokens, table.t(), V, 1.0, X), (tokens.cpu(), table, V, 1.0, X)):
        with pytest.raises(symi.SymiError):
            symi.symi_embed_fwd(ctx, *bad)
    for bad in ((tokens, X, V, 1.0, 2, dT, ws), (tokens, X, 0, 1.0, 0, dT, ws), (tokens, X, V, 1.0, 0, dT.to(torch.bfloat16), ws),
                (tokens, X, V, 1.0, 0, dT[:-1], ws), (tokens, X, V, 1.0, 0, dT, ws[:-1]), (tokens, X.float(), V, 1.0, 0, dT, ws)):
        with pytest.raises(symi.SymiError):
            symi.symi_embed_bwd(ctx, *bad)
    L = symi.lib()
    assert L.symi_embed_fwd(ctx.ptr, None, None, V, 1.0, None, None) == -1 and "NULL" in symi.symi_last_error()
    assert L.symi_embed_bwd(ctx.ptr, None, None, V, 1.0, 0, None, None, None) == -1
    assert L.symi_embed_fwd(None, None, None, V, 1.0, None, None) == -1
