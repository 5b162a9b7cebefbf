"""Batches on both sides of the number of rows from which on rows are not split over workgroups: the same bits, row by row."""
import pytest
import torch

import paper_2504_19925_amd as symi
from tests.test_gpu_policy import HIGH, KL, LOW, batch, call, context

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pieces,waves", [(500, 2), (1000, 4), (1500, 4), (2000, 4), (2500, 8), (3000, 8), (4000, 8), (6250, 8), (8192, 8), (10000, 16), (16384, 16)])
def test_the_same_bits_on_both_sides(pieces, waves, dtype):
    V = pieces * (8 if dtype == "bf16" else 4)
    units = torch.cuda.get_device_properties(0).multi_processor_count
    each = 58000 if waves == 8 and dtype == "f32" else 80000
    line = min(256, 4 * units // waves, 10 ** 9 if waves == 16 else waves * each // pieces)
    hp = symi.SymiPolicy.make(LOW, HIGH, KL, 1.0, 1.0, dtype)
    small = batch(3, V, V, dtype, pieces)
    small["weight"].fill_(0.5)
    few = call(context(3), hp, small, V)
    for T in (line - 1, line, line + 1, line + 2):
        many = {k: torch.cat([v] * -(-T // 3))[:T].contiguous() for k, v in small.items()}
        logp, _, dz = call(context(T), hp, many, V)
        at = torch.arange(T, device="cuda") % 3
        assert torch.equal(logp, few[0][at]) and torch.equal(dz, few[2][at]), T
