"""The embedding gradient's ways through a batch: no sort (few tokens), the sort's kept tokens and its second reading, rows of the table
beyond one workgroup's, chunks of every length, long runs and their shares, zeros in both launches.

Against sums in binary64 with the bound of test_gpu_embed.py: n + 2 roundings of at most the sum of the summands' sizes."""
import numpy as np
import pytest
import torch

import harness as Hn
from tests.test_gpu_embed import U32, backward, context, gen, make_tokens

pytestmark = pytest.mark.gpu


def sums(tokens, dX, V, scale):
    """Rows' sums, sums of sizes and counts, on the CPU: rows sorted, one addition after the other (a GPU's additions of 64-bit values to
    one address take turns, millions of them for minutes)."""
    t = tokens.cpu().numpy().astype(np.int64)
    live = np.nonzero((t >= 0) & (t < V))[0]
    live = live[np.argsort(t[live], kind="stable")]
    n = np.bincount(t[live], minlength=V)
    want, size = np.zeros((V, dX.shape[1])), np.zeros((V, dX.shape[1]))
    if len(live):
        x = Hn.npf(dX)[live].astype(np.float64) * scale
        rows = np.nonzero(n)[0]
        starts = (np.cumsum(n) - n)[rows]
        want[rows] = np.add.reduceat(x, starts, axis=0)
        size[rows] = np.add.reduceat(np.abs(x, out=x), starts, axis=0)
    return [torch.from_numpy(a).cuda() for a in (want, size, n.astype(np.float64))]


def check(reference, got, old=None):
    want, size, n = reference
    if old is not None:
        assert torch.equal(got[n == 0], old[n == 0])
        want, size = want + old.double(), size + old.double().abs()
    # the reference's own sums are off by 2^-53 for each of their terms
    assert ((got.double() - want).abs() <= (n + 2)[:, None] * U32 * size).all()


CASES = [  # T, d, V, tokens
    (64, 70000, 9, "few"), (65, 4096, 300, "skewed"), (512, 4096, 300, "uniform"), (513, 4096, 300, "skewed"), (512, 8, 1000, "same"),
    (2048, 1024, 77, "skewed"), (2048, 1032, 77, "skewed"), (2049, 512, 5000, "padded"), (2048, 8, 20000, "uniform"),
    (4096, 2056, 3000, "skewed"), (8191, 520, 1, "same"), (8193, 520, 257, "uniform"), (20000, 264, 2, "uniform"), (20000, 2048, 100003, "skewed"),
    (30000, 72, 70001, "padded"), (65536, 8, 300, "same"), (65536, 1024, 999, "skewed"), (70000, 16, (1 << 18) + 77, "padded"),
    (70001, 24, (1 << 19) - 1, "few"), (131072, 40, 64, "uniform"), ((1 << 22) + 5, 8, 1000, "skewed"), (16385, 4096, 5000, "skewed")]


# a context takes fp32 batches of up to 2^22 - 4 k tokens
@pytest.mark.parametrize("T,d,V,kind,dtype", [(*c, t) for c in CASES for t in ("bf16", "f32") if t == "bf16" or c[0] <= 1 << 20])
def test_paths(T, d, V, kind, dtype):
    print(f"[embed] {dtype} T={T} d={d} V={V} {kind}", flush=True)
    ctx = context(T, d, dtype)
    tokens = make_tokens(kind, T, V, T + d)
    dX = torch.randn(T, d, generator=gen(T), device="cuda").to(ctx.torch_dtype)
    got = backward(ctx, tokens, dX, V, 0.75)
    print("[embed] the reference", flush=True)
    reference = sums(tokens, dX, V, 0.75)
    check(reference, got)
    assert torch.equal(got, backward(ctx, tokens, dX, V, 0.75))
    old = torch.randn(V, d, generator=gen(1), device="cuda")
    added = backward(ctx, tokens, dX, V, 0.75, old)
    check(reference, added, old)


def test_a_frequent_row_beside_rare_ones():
    """One row with a quarter of the batch, one with a run of every length around the chunks', the others once."""
    T, d, V = 65536, 264, 40000
    ctx = context(T, d, "bf16")
    tokens = torch.arange(T, device="cuda") % 20000 + 20000
    tokens[::4] = 7
    at = 1
    for run in range(1, 140):
        tokens[torch.arange(run, device="cuda") * 4 + at] = 100 + run
        at += run * 4
        at += (1 - at) % 4
    tokens = tokens[torch.randperm(T, generator=gen(3), device="cuda")].to(torch.int32)
    dX = torch.randn(T, d, generator=gen(4), device="cuda").to(torch.bfloat16)
    check(sums(tokens, dX, V, 1.0), backward(ctx, tokens, dX, V, 1.0))
