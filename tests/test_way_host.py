"""The way into the experts without a GPU: sizes, refusals, and the oracle's own pins."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2504_19925_amd as symi
from oracle import way_oracle as O


def _cfg(T=100, E=8, k=2, d=64, f=96, S=8, dtype="bf16", renorm=1):
    return symi.SymiCfg.make(T, E, k, d, f, S, 1, 0, dtype, renorm)


def test_sizes():
    assert [symi.symi_pitch8(n) for n in (8, 128, 136, 1 << 22)] == [128, 128, 256, 1 << 22]
    assert [symi.symi_scale_pitch8(n) for n in (8, 512, 520, 1 << 22)] == [4, 4, 8, 1 << 15]
    for n in (0, -8, 4, 12, (1 << 22) + 8):
        for call in (symi.symi_pitch8, symi.symi_scale_pitch8):
            with pytest.raises(symi.SymiError, match="multiple of 8"):
                call(n)
    for call in (symi.symi_norm_workspace_bytes, symi.symi_workspace8_bytes):
        assert call(_cfg()) > 0 and call(_cfg(T=0)) > 0 and call(_cfg(T=-1)) == 0 and symi.symi_last_error()
    # every row of both operands, and its scales
    assert symi.symi_workspace8_bytes(_cfg(T=1000)) > 2000 * (128 + 4 + 128 + 4)


def test_device_calls_refuse_cpu_tensors_and_missing_contexts():
    ctx = symi.SymiCtx(None, _cfg(), 0)
    x, row, i = torch.zeros(100, 64, dtype=torch.bfloat16), torch.zeros(100), torch.zeros(200, dtype=torch.int32)
    with pytest.raises(symi.SymiError, match="X"):
        symi.symi_norm_fwd(ctx, 1, 1e-5, x, None, None, None, None, x, None, None)
    with pytest.raises(symi.SymiError, match="dY"):
        symi.symi_norm_bwd(ctx, 1, x, x, row, row, None, None, x, None, None, x)
    with pytest.raises(symi.SymiError, match="logits"):
        symi.symi_route_scored(ctx, symi.SymiScore.make(), torch.zeros(100, 8), None, i, row, i)
    with pytest.raises(symi.SymiError, match="X"):
        symi.symi_quant8(ctx, x, 1, 100, 64, 1, x, x)
    L, hp = symi.lib(), symi.SymiScore.make()
    for name, args in (("symi_norm_fwd", 12), ("symi_norm_bwd", 13), ("symi_route_scored", 8), ("symi_route_scored_bwd", 8), ("symi_route_bias", 5),
                       ("symi_quant8", 9), ("symi_dequant8", 9), ("symi_product8", 11), ("symi_expert_fwd8", 12)):
        fn = getattr(L, name)
        assert len(fn.argtypes) == args
        zeros = [None if t in (ctypes.c_void_p,) else ctypes.byref(hp) if t == ctypes.POINTER(symi.SymiScore) else 0 for t in fn.argtypes]
        assert fn(*zeros) == -1 and "ctx" in symi.symi_last_error(), name


def test_oracle_norm_gradient_is_that_of_its_norm():
    rng = np.random.default_rng(1)
    T, d = 3, 16
    R, w, b, dY = rng.standard_normal((T, d)), rng.standard_normal(d), rng.standard_normal(d), rng.standard_normal((T, d))
    for center in (0, 1):
        n = O.norm(R, center, 1e-3, w, b)
        got = O.norm_gradient(dY, R, n["mean"], n["rstd"], center, w)
        loss = lambda R, w, b: (O.norm(R, center, 1e-3, w, b)["Y"] * dY).sum()   # noqa: E731
        for x, g, at in ((R, got["dX"], 0), (w, got["dw"], 1), (b, got["db"], 2)):
            for i in np.ndindex(*x.shape):
                h = np.zeros_like(x)
                h[i] = 1e-6
                up, down = [R, w, b], [R, w, b]
                up[at], down[at] = x + h, x - h
                assert abs((loss(*up) - loss(*down)) / 2e-6 - g[i]) < 1e-7


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renorm", [0, 1])
def test_oracle_route_gradient_is_that_of_its_gates(sigmoid, renorm):
    rng = np.random.default_rng(2)
    z, bias, dg = rng.standard_normal((4, 12)) * 2, rng.standard_normal(12) * 0.1, rng.standard_normal((4, 3))
    z[1, 4:] = -np.inf
    z[2, 2:] = -np.inf          # one class fills up
    args = (bias, 3, renorm, sigmoid, 3, 2, 2, 1.7)
    r = O.route(z, *args)
    assert r["real"].sum(axis=1).tolist() == [3, 3, 2, 3] and r["gate"][2, 2] == 0 and r["idx"][2, 2] == 2
    got, size = O.route_gradient(z, r["idx"], r["real"], dg, renorm, sigmoid, 1.7)
    assert (size >= np.abs(got) - 1e-15).all()
    for t in range(4):
        for e in range(12):
            if z[t, e] == -np.inf:
                assert got[t, e] == 0
                continue
            h = np.zeros_like(z)
            h[t, e] = 1e-6
            up, down = O.route(z + h, *args), O.route(z - h, *args)
            assert (up["idx"] == r["idx"]).all() and (down["idx"] == r["idx"]).all()
            assert abs(((up["gate"] - down["gate"]) * dg).sum() / 2e-6 - got[t, e]) < 1e-7


def test_oracle_codes_are_those_of_e4m3():
    """Powers and roundings against torch's own cast to e4m3, which rounds to nearest even."""
    rng = np.random.default_rng(3)
    x = (rng.standard_normal((20, 300)) * np.exp(4 * rng.standard_normal((20, 1)))).astype(np.float32)
    x[3] = 0
    x[4, :128] *= 1e-30
    x[5, 7] = 448.0 * 2 ** 5
    x[6, 9] = np.nextafter(np.float32(448.0 * 2 ** 5), np.float32(np.inf))
    x[7, 100:130] = 2.0 ** -140
    for block in (1, 128):
        q, s = O.quant(x, block)
        scale = np.repeat(np.repeat(2.0 ** (s - 127.0), block, axis=0)[:20], 128, axis=1)[:, :300]
        assert np.abs(q).max() <= 448 and (np.abs(x) <= 448 * scale).all()
        tight = np.repeat(np.repeat(s > 0, block, axis=0)[:20], 128, axis=1)[:, :300]
        if block == 1:
            most = np.pad(np.abs(x), ((0, 0), (0, 84))).reshape(20, 3, 128).max(axis=2)
            assert (most[s > 0] > 224 * 2.0 ** (s[s > 0] - 127.0)).all() and tight.any()
        want = torch.from_numpy((x.astype(np.float64) / scale).astype(np.float32)).to(torch.float8_e4m3fn).float().numpy()
        assert (want == q).all()
    assert O.power(448.0) == 127 and O.power(448.0001) == 128 and O.power(0.0) == 0 and O.power(2.0 ** -149) == 0
