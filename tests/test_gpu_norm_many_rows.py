"""Norms and their gradients over more rows than a launch has at once, so that every form goes on to further rows, and over as many as a launch needs a second
dimension for.  Oracle and bounds are those of the norms' other tests."""
import numpy as np
import pytest
import torch

import harness as Hn
import paper_2504_19925_amd as symi
from tests.test_gpu_norm import EPS, U32, check_gradient, check_norm, context, randn, rows, statistics

pytestmark = pytest.mark.gpu

# threads of a row x pieces of 8 values each: 16 x 1, 16 x 2, 64 x 1, 64 x 2, 128 x 2, 512 x 1, 512 x 2, 1024 x 2, full and ragged rows
FORWARD = [(60001, 72), (30001, 256), (15001, 456), (7001, 1024), (7001, 520), (3501, 2048), (3501, 1160), (1701, 4096), (1701, 2056), (601, 8192), (601, 4104),
           (601, 16384), (601, 8200)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", FORWARD)
def test_norm(T, d, dtype):
    ctx = context(T, d, dtype)
    dt = ctx.torch_dtype
    w, b = 1 + 0.3 * randn(10, d), 0.2 * randn(11, d)
    X, res = rows(30, T, d, dt), rows(20, T, d, dt)
    for center, r in ((0, None), (1, res)):
        print(f"[norm] {dtype} T={T} d={d} center={center} residual={r is not None}", flush=True)
        R, Y, mean, rstd, _ = check_norm(ctx, center, EPS, X.clone(), r, w, b)
        # the last rows, alone
        few = context(7, d, dtype)
        R2, Y2, m2, s2, _ = check_norm(few, center, EPS, X[-7:].clone(), None if r is None else r[-7:].contiguous(), w, b)
        assert torch.equal(Y[-7:], Y2) and torch.equal(rstd[-7:], s2) and torch.equal(mean[-7:], m2) and (r is None or torch.equal(R[-7:], R2))


# partial sums of dw and db in every form: more than 768 rows, of more than 2048 values more than 2560
GRADIENT = [(9001, 128), (2100, 200), (9001, 456), (3001, 1024), (2001, 520), (3001, 2048), (2700, 4096), (2600, 2056), (2600, 8192), (2601, 4104)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", GRADIENT)
def test_gradient(T, d, dtype):
    ctx = context(T, d, dtype)
    dt = ctx.torch_dtype
    w = 1 + 0.3 * randn(10, d)
    R, dY, dR = rows(1, T, d, dt), randn(2, T, d).to(dt), randn(3, T, d).to(dt)
    for center, r in ((1, dR), (0, None)):
        print(f"[norm gradient] {dtype} T={T} d={d} center={center} dR={r is not None}", flush=True)
        mean, rstd = statistics(R, center)
        first = check_gradient(ctx, center, dY, R, mean, rstd, w, r)
        into = dY.clone()
        again = check_gradient(ctx, center, into, R, mean, rstd, w, r, into=into)
        assert all(torch.equal(x, y) for x, y in zip(first, again))


def few_of_many(T, d, seed, at):
    """T rows of zeros but for those at `at`."""
    X = torch.zeros(T, d, dtype=torch.bfloat16, device="cuda")
    X[at] = rows(seed, len(at), d, torch.bfloat16)
    return X


def only_at(X, at):
    """Whether all other rows are zeros; a gigabyte at a time."""
    kept = X[at].clone()
    X[at] = 0
    empty = not any(x.any() for x in X.view(-1).split(1 << 29))
    X[at] = kept
    return empty


def test_wide_rows_in_two_dimensions_of_a_launch():
    """Rows that do not stay in registers, a workgroup each: 2^20 of them and more."""
    torch.cuda.empty_cache()
    T, d = (1 << 20) + 3, 16392
    at = [0, 1, (1 << 20) - 1, 1 << 20, T - 1]
    ctx, few = context(T, d, "bf16"), context(len(at), d, "bf16")
    X, w = few_of_many(T, d, 1, at), 1 + 0.3 * randn(10, d)
    Y, mean, rstd = torch.ones_like(X), torch.full((T,), float("nan"), device="cuda"), torch.full((T,), float("nan"), device="cuda")
    print(f"[norm] T={T} d={d}", flush=True)
    symi.symi_norm_fwd(ctx, 1, EPS, X, None, w, None, None, Y, mean, rstd)
    _, Y2, m2, s2, _ = check_norm(few, 1, EPS, X[at].contiguous(), None, w, None)
    assert torch.equal(Y[at], Y2) and torch.equal(mean[at], m2) and torch.equal(rstd[at], s2)
    assert only_at(Y, at) and not torch.isnan(mean).any() and not torch.isnan(rstd).any()


def test_gradient_of_more_wide_rows_than_one_dimension_of_a_launch_has():
    """It ends at 2^32 threads, which 2^22 rows of a workgroup of 1024 each reach.  In place, so that it is two tensors of 69 GB."""
    torch.cuda.empty_cache()
    T, d = (1 << 22) + 3, 8200
    at = [0, 1, (1 << 20) - 1, 1 << 20, (1 << 22) - 1, 1 << 22, T - 1]
    ctx, few = context(T, d, "bf16"), context(len(at), d, "bf16")
    R, dY, w = few_of_many(T, d, 1, at), few_of_many(T, d, 5, at), 1 + 0.3 * randn(10, d)
    mean, rstd = torch.zeros(T, device="cuda"), torch.ones(T, device="cuda")
    mean[at], rstd[at] = statistics(R[at].contiguous(), 1)
    parts = [t[at].contiguous() for t in (dY, R, mean, rstd)]
    want = check_gradient(few, 1, *parts, w, None)
    dw, db = torch.full((d,), float("nan"), device="cuda"), torch.full((d,), float("nan"), device="cuda")
    ws = torch.full((symi.symi_norm_workspace_bytes(ctx),), 0xA5, dtype=torch.uint8, device="cuda")
    print(f"[norm gradient] T={T} d={d}", flush=True)
    symi.symi_norm_bwd(ctx, 1, dY, R, mean, rstd, w, None, dY, dw, db, ws)
    assert torch.equal(dY[at], want[0]) and only_at(dY, at)
    # the same summands, in an order of their own
    xh = (Hn.npf(parts[1]).astype(np.float64) - Hn.npf(parts[2])[:, None]) * Hn.npf(parts[3])[:, None].astype(np.float64)
    dy = np.abs(Hn.npf(parts[0]).astype(np.float64))
    assert (np.abs(Hn.npf(dw) - Hn.npf(want[1])) <= 2 * (len(at) + 4) * U32 * 1.05 * (dy * np.abs(xh)).sum(axis=0)).all()
    assert (np.abs(Hn.npf(db) - Hn.npf(want[2])) <= 2 * (len(at) + 4) * U32 * 1.05 * dy.sum(axis=0)).all()
