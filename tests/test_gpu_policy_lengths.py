"""The clipped policy loss on both sides of every length and batch at which its workgroups change, rows beginning anywhere:
against binary64, with the bounds of test_gpu_policy.py, and the same bits for a row in any batch."""
import numpy as np
import pytest
import torch

import paper_2504_19925_amd as symi
from tests.test_gpu_policy import HIGH, KL, LOW, batch, call, check, context

pytestmark = pytest.mark.gpu
PIECES = [63, 64, 255, 256, 257, 511, 512, 513, 1023, 1024, 1025, 2047, 2048, 2049, 2999, 3000, 3001, 4607, 4608, 4609, 8191, 8192, 8193,
          12800, 12801, 16383, 16384, 16385, 24577]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pieces", PIECES)
def test_every_length(pieces, dtype):
    n = 8 if dtype == "bf16" else 4
    hp = symi.SymiPolicy.make(LOW, HIGH, KL, 0.9, 1.0, dtype)
    for V, ld in ((pieces * n, pieces * n), (pieces * n, pieces * n + 1), (pieces * n - 1, pieces * n - 1), (pieces * n + 3, pieces * n + 8)):
        print(f"[policy] {dtype} pieces={pieces} V={V} ld={ld}", flush=True)
        T = 9
        b = batch(T, V, ld, dtype, pieces)
        b["weight"][::2] += 0.1
        b["action"][0], b["action"][2] = 0, V - 1             # the ends of a row
        lp = torch.log_softmax(b["z"][:, :V].double() * hp.inv_temperature, 1).gather(1, b["action"].long()[:, None])[:, 0]
        b["old"] = (lp - 0.1).float()
        b["ref"] = (lp + 0.1).float()
        out = call(context(T), hp, b, V)
        check(b, V, hp, *out)
        # the loss alone
        check(b, V, hp, *call(context(T), hp, b, V, grad=False)[:2], None)


@pytest.mark.parametrize("V,ld", [(2100, 2112), (8184, 8184), (16392, 16400), (28000, 28000), (40000, 40000), (65528, 65528), (70008, 70016)])
def test_a_row_has_the_same_bits_in_any_batch(V, ld):
    """Few rows are split over workgroups, many are not; nine times the same three rows between others.  Rows of 16 bytes' multiples."""
    hp = symi.SymiPolicy.make(LOW, HIGH, KL, 1.0, 1.0, "bf16")
    small = batch(3, V, ld, "bf16", 5)
    small["weight"].fill_(0.5)
    few = call(context(3), hp, small, V)
    for T in (65, 129, 257, 600):
        many = {k: torch.cat([v] * -(-T // 3))[:T].contiguous() for k, v in small.items()}
        logp, stats, dz = call(context(T), hp, many, V)
        for i in range(T):
            if i % 37 < 3:
                assert torch.equal(logp[i], few[0][i % 3]) and torch.equal(dz[i], few[2][i % 3]), (T, i)
        want = few[1].double() * T / 3
        if T % 3 == 0:
            assert ((stats.double() - want).abs() <= 2.0 ** -23 * T / 3 * few[1].double().abs() + 1e-12).all()


def test_a_table_of_rows_around_other_memory():
    """Odd rows in the middle of a buffer: what lies before and behind the gradient stays."""
    for dtype, dt in (("bf16", torch.bfloat16), ("f32", torch.float32)):
        hp = symi.SymiPolicy.make(LOW, HIGH, KL, dtype=dtype)
        for V, ld in ((4493, 4493), (13, 13), (9, 11), (1, 1)):
            T = 20
            b = batch(T, V, ld, dtype, 3)
            whole = torch.full((T * ld + 32,), 7.0, dtype=dt, device="cuda")
            for by in (1, 7, 16):
                whole.fill_(7.0)
                out = whole[by:by + T * ld].view(T, ld)
                check(b, V, hp, *call(context(T), hp, b, V, out=out))
                assert (whole[:by] == 7).all() and (whole[by + T * ld:] == 7).all()
