"""Routing by scores in every form that a batch can take: lanes of a token times pieces of 4 classes a lane.  A token has the same bits in all of them, those of
one piece a lane (small batches), which are compared with binary64 in the routing's other tests; here a sample of the tokens is as well."""
import numpy as np
import pytest
import torch

import harness as Hn
import paper_2504_19925_amd as symi
from oracle import way_oracle as O
from tests.test_gpu_scored import U32, bound_of, context, gen, run

pytestmark = pytest.mark.gpu


def form(E, T):
    """(lanes, pieces), by the library's rule."""
    vecs, G = -(-E // 4), 1
    while G * 4 < vecs:
        G *= 2
    while G < vecs and G < 64 and T * G < 512 * 256:
        G *= 2
    need = -(-vecs // G)
    return G, 1 if need <= 1 else 2 if need <= 2 else 4


# E, T of the largest batch, smaller ones, groups, top_groups, k, the forms
CASES = [
    (4, 131072, (65536,), 2, 1, 2, {(1, 1)}),
    (8, 131072, (70000, 900), 4, 2, 3, {(1, 2), (2, 1)}),
    (12, 131075, (70000, 900), 3, 2, 3, {(1, 4), (2, 2), (4, 1)}),
    (16, 131073, (65537, 900), 4, 3, 4, {(1, 4), (2, 2), (4, 1)}),
    (20, 65600, (40000, 900), 5, 3, 6, {(2, 4), (4, 2), (8, 1)}),
    (32, 66000, (33000, 900), 8, 3, 6, {(2, 4), (4, 2), (8, 1)}),
    (64, 40000, (17000, 900), 8, 4, 6, {(4, 4), (8, 2), (16, 1)}),
    (64, 40000, (17000,), 2, 1, 6, {(4, 4), (8, 2)}),
    (60, 33000, (17000, 900), 6, 2, 8, {(4, 4), (8, 2), (16, 1)}),
    (128, 40001, (9000, 900), 8, 4, 8, {(8, 4), (16, 2), (32, 1)}),
    (128, 17000, (9000,), 32, 5, 16, {(8, 4), (16, 2)}),
    (200, 8300, (4500, 3000, 900), 10, 4, 9, {(16, 4), (32, 2), (64, 1)}),
    (256, 8300, (4500, 900), 4, 2, 8, {(16, 4), (32, 2), (64, 1)}),
    (512, 4500, (900,), 64, 20, 16, {(32, 4), (64, 2)}),
    (1000, 4500, (900,), 8, 3, 7, {(64, 4)}),
]


def oracle_agrees(z, bias, idx, gate, at, k, renorm, score, groups, top_groups, group_top, scale):
    z64 = Hn.npf(z[at])
    want = O.route(z64, None if bias is None else Hn.npf(bias), k, renorm, score == "sigmoid", groups, top_groups, group_top, float(np.float32(scale)))
    assert (Hn.npf(idx[at]) == want["idx"]).all()
    tol = bound_of(z64, want["idx"], want["real"], score == "sigmoid")
    assert (np.abs(Hn.npf(gate[at]) - want["gate"]) <= tol * np.abs(want["gate"]) + 2.0 ** -140).all()
    return want, z64, tol


@pytest.mark.parametrize("E,T,smaller,groups,top_groups,k,forms", CASES, ids=lambda x: str(x) if isinstance(x, int) else None)
@pytest.mark.parametrize("score,renorm", [("softmax", 0), ("softmax", 1), ("sigmoid", 0), ("sigmoid", 1)])
def test_a_token_has_the_same_bits_in_every_form(E, T, smaller, groups, top_groups, k, forms, score, renorm):
    assert {form(E, n) for n in (T, *smaller)} == forms
    g = gen(E + T)
    z = torch.randn(T, E, generator=g, device="cuda") * torch.exp(0.5 * torch.randn(T, 1, generator=g, device="cuda"))
    z[torch.rand(T, E, generator=g, device="cuda") < 0.03] = -float("inf")
    z[3::97] = torch.randint(-2, 3, z[3::97].shape, generator=g, device="cuda").float()                                # equal values
    z[5::89] = 0.25 + torch.randint(-3, 4, z[5::89].shape, generator=g, device="cuda") * 2.0 ** -25                    # a rounding apart
    z[7::101] = -float("inf")
    bias = 0.1 * torch.randn(E, generator=g, device="cuda")
    everywhere = {0, 1, T - 1, *torch.randint(0, T, (150,), generator=gen(2), device="cuda").tolist(), *range(3, T, 97 * (T // 2000)), *range(5, T, 89 * (T // 2000)),
                  *range(7, T, 101 * (T // 2000))}
    per = E // groups
    for b, group_top, grouped in ((bias, min(2, per), True), (None, min(2, per), True), (bias, 1, False), (None, 1, True)):
        gr, tg = (groups, top_groups) if grouped else (1, 1)
        print(f"[scored forms] E={E} T={T} {smaller} {score} renorm={renorm} bias={b is not None} {gr}/{tg}/{group_top}", flush=True)
        hp = symi.SymiScore.make(score, gr, tg, group_top, 1.75)
        idx, gate, hist = run(context(T, E, k, renorm), hp, z, b)
        assert torch.equal(hist.long(), torch.bincount(idx.view(-1).long(), minlength=E))
        # sums of two scores a rounding apart are nearer to each other than binary64's own rounding: those rows are compared between the forms only
        sample = sorted(t for t in everywhere if b is not None or group_top == 1 or t % 89 != 5)
        want, z64, tol = oracle_agrees(z, b, idx, gate, sample, k, renorm, score, gr, tg, group_top, 1.75)
        for n in smaller:
            for first in {0, (T - n) // 2 + 1, T - n}:
                few = run(context(n, E, k, renorm), hp, z[first:first + n].contiguous(), b)
                assert torch.equal(few[0], idx[first:first + n]) and torch.equal(few[1], gate[first:first + n])
        dgate = torch.randn(T, k, generator=gen(77), device="cuda")
        dz = torch.full_like(z, float("nan"))
        symi.symi_route_scored_bwd(context(T, E, k, renorm), hp, z, idx, gate, dgate, dz)
        grad, size = O.route_gradient(z64, want["idx"], want["real"], Hn.npf(dgate[sample]), renorm, score == "sigmoid", float(np.float32(1.75)))
        assert (np.abs(Hn.npf(dz[sample]) - grad) <= (3 * tol + 32 * U32) * size + 2.0 ** -140).all()
        n = smaller[-1]
        few = torch.full((n, E), float("nan"), device="cuda")
        symi.symi_route_scored_bwd(context(n, E, k, renorm), hp, z[-n:].contiguous(), idx[-n:].contiguous(), gate[-n:].contiguous(), dgate[-n:].contiguous(), few)
        assert torch.equal(few, dz[-n:])
