"""The ends of the step without a GPU: workspace sizes, refusals of the host functions, and the oracle's own pins."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2504_19925_amd as symi
from paper_2504_19925_amd.binding import SymiAdamWTensor
from oracle import ends_oracle as O


def _cfg(T=100, d=64, dtype="bf16"):
    return symi.SymiCfg.make(T, 1, 1, d, 8, 1, 1, 0, dtype)


def test_workspace_sizes():
    assert symi.symi_embed_workspace_bytes(_cfg(), 1000) > 0 and symi.symi_policy_workspace_bytes(_cfg()) > 0
    assert symi.symi_embed_workspace_bytes(_cfg(), 0) == 0 and "V" in symi.symi_last_error()
    assert symi.symi_embed_workspace_bytes(_cfg(d=12), 10) == 0 and symi.symi_policy_workspace_bytes(_cfg(T=-1)) == 0
    assert symi.symi_embed_workspace_bytes(_cfg(), 2 ** 31 - 1) > 4 * (2 ** 31 - 1)
    assert symi.symi_embed_workspace_bytes(_cfg(T=0), 5) > 0


def test_descriptions_are_checked_before_any_device_is_needed():
    L = symi.lib()
    out = ctypes.c_void_p()
    ok = dict(param=8, grad=8, m=8, v=8, n=10, decay=1.0, state_bits=32)      # never read: refused first

    def create(count=1, **kw):
        t = (SymiAdamWTensor * 1)(SymiAdamWTensor(**{**ok, **kw}))
        size = L.symi_adamw_table_bytes(t, count)
        rc = L.symi_adamw_create(t, count, 256, ctypes.byref(out), None)
        assert (size > 0) == (rc not in (-1, -2))
        return rc

    assert L.symi_adamw_create(None, 1, None, ctypes.byref(out), None) == -1 and L.symi_adamw_create(None, 0, None, None, None) == -1
    assert L.symi_adamw_create((SymiAdamWTensor * 1)(SymiAdamWTensor(**ok)), 1, None, ctypes.byref(out), None) == -1   # no table
    for kw in (dict(n=-1), dict(state_bits=16), dict(param_dtype=2), dict(grad_dtype=-1), dict(decay=-1.0), dict(decay=float("nan")),
               dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(param_dtype=1), dict(master=8), dict(state_bits=8),
               dict(state_bits=8, m_scale=8), dict(m_scale=8), dict(v_scale=8), dict(count=-1)):
        assert create(**kw) == -1, kw
        assert not out.value and symi.symi_last_error()
    assert create(n=2 ** 37) == -2 and create(n=2 ** 62) == -2
    assert L.symi_adamw_destroy(None) == 0 and L.symi_adamw_values(None) == 0
    if not torch.cuda.is_available():
        assert create() == -3 and not out.value


def test_device_calls_refuse_cpu_tensors():
    ctx = symi.SymiCtx(None, _cfg(), 0)
    z, i = torch.zeros(100, 64, dtype=torch.bfloat16), torch.zeros(100, dtype=torch.int32)
    with pytest.raises(symi.SymiError, match="tokens"):
        symi.symi_embed_fwd(ctx, i, z, 100, 1.0, z)
    with pytest.raises(symi.SymiError, match="logits"):
        symi.symi_token_logp(ctx, symi.SymiPolicy.make(), z, 64, 64, i, None, torch.zeros(100))
    with pytest.raises(symi.SymiError, match="tensor 0"):
        symi.symi_adamw_create([dict(param=torch.zeros(3), grad=torch.zeros(3), m=torch.zeros(3), v=torch.zeros(3))])


def test_oracle_policy_gradient_is_that_of_its_loss():
    rng = np.random.default_rng(1)
    T, V = 6, 11
    z, A, w = rng.standard_normal((T, V)) * 2, rng.standard_normal(T), rng.random(T)
    a = rng.integers(0, V, T)
    w[2], a[3] = 0, -1
    lp = np.array([z[t] - z[t].max() - np.log(np.exp(z[t] - z[t].max()).sum()) for t in range(T)])[np.arange(T), a]
    old, ref = lp + np.array([0.05, -0.6, 0.0, 0.1, 0.5, -0.1]), lp + 0.3 * rng.standard_normal(T)
    run = lambda x: O.policy(x, V, a, old, ref, A, w, 0.2, 0.3, 0.1, 0.7, 1.0)   # noqa: E731
    got = run(z)["dlogits"]
    assert not got[2].any() and not got[3].any() and np.abs(got.sum(axis=1)).max() < 1e-12
    for t in range(T):
        for j in range(V):
            d = np.zeros_like(z)
            d[t, j] = 1e-6
            assert abs((run(z + d)["stats"][0] - run(z - d)["stats"][0]) / 2e-6 - got[t, j]) < 1e-7


def test_oracle_codes():
    """Codes stand for what they say, are neighbours of the value, and mean it."""
    rng = np.random.default_rng(2)
    x = np.abs(rng.standard_normal(256)) * 10 ** rng.uniform(-6, 0, 256)
    for power, top in ((2, 127), (4, 255)):
        mean = np.zeros(256)
        for u in (np.arange(1000) + 0.5) / 1000:
            code, _ = O.encode(x, power, top, u)
            value = (code / top) ** power * x.max()
            mean += value / 1000
            assert (np.abs(value - x) <= ((code + 1) ** power - np.maximum(code - 1, 0) ** power) / top ** power * x.max()).all()
        assert np.abs(mean - x).max() <= 1e-3 * power / top * x.max() + 1e-12
    um, uv = O.random_numbers(3, 4, 5, 100000)
    assert 0 < um.min() and um.max() < 1 and abs(um.mean() - 0.5) < 0.005 and abs(np.corrcoef(um, uv)[0, 1]) < 0.02
    assert (O.random_numbers(3, 4, 6, 256)[0] == um[256:512]).all() and (O.random_numbers(3, 5, 5, 256)[0] != um[:256]).mean() > 0.99
