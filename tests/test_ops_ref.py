"""The plain forms' written-out gradients against automatic differentiation of the definitions and
against differences, in 64 bits (CPU)."""
import math

import pytest
import torch

import ops_ref as R


def rnd(*s, seed=0):
    return torch.randn(*s, dtype=torch.float64, generator=torch.Generator().manual_seed(seed + sum(s)))


def differences(f, v, eps=1e-6):
    out = torch.zeros_like(v)
    for i in range(v.numel()):
        d = torch.zeros(v.numel(), dtype=v.dtype)
        d[i] = eps
        d = d.view(v.shape)
        out.view(-1)[i] = (f(v + d) - f(v - d)) / (2 * eps)
    return out


@pytest.mark.parametrize("renorm", [False, True])
def test_route_gradient(renorm):
    l = rnd(5, 9, seed=3)
    l[1, 4] = -math.inf
    l[2, 1:] = -math.inf  # one expert for three slots
    mask = torch.tensor([1, 1, 1, 0, 1])
    dw = rnd(5, 3, seed=4)
    idx, w, p = R.route(l, 3, renorm, mask)
    counts, mean, coef, loss = R.balance(idx, p, 3, 0.3, mask)
    assert int(counts.sum()) == 10 and idx[2].tolist() == [0, -1, -1] and idx[3].tolist() == [-1] * 3

    def total(x):
        i2, w2, p2 = R.route(x, 3, renorm, mask)
        assert torch.equal(i2, idx)
        return 0.7 * (coef * p2.sum(0)).sum() + (w2 * dw).sum()

    got, mag = R.route_bwd(idx, w, p, renorm, dw, coef, 0.7)
    fin = l.masked_fill(l == -math.inf, 0.0)
    want = differences(lambda x: total(x.masked_fill(l == -math.inf, -math.inf)), fin)
    assert torch.allclose(got, want.masked_fill(l == -math.inf, 0.0), atol=1e-8) and bool((mag >= got.abs() - 1e-15).all())
    assert math.isclose(float((coef * p.sum(0)).sum()), float(loss), rel_tol=1e-12)


@pytest.mark.parametrize("gate", [None, "channel", "token"])
@pytest.mark.parametrize("post,pre", [(True, True), (True, False), (False, True), (False, False)])
def test_block_norm_gradient(gate, post, pre):
    t, h = 3, 6
    v = {"x": rnd(t, h), "y": rnd(t, h, seed=1), "g_post": rnd(h) if post else None,
         "gate": {None: None, "channel": rnd(h, seed=2), "token": rnd(t, 1, seed=2)}[gate], "g_pre": rnd(h, seed=5) if pre else None}
    dxo, dh = rnd(t, h, seed=6), rnd(t, h, seed=7) if pre else None

    def total(**k):
        u = {**v, **k}
        xo, hh, _ = R.block_norm(u["x"], u["y"], u["g_post"], u["gate"], 0.8, u["g_pre"], 1e-3)
        return (xo * dxo).sum() + (0 if hh is None else (hh * dh).sum())

    xo = R.block_norm(v["x"], v["y"], v["g_post"], v["gate"], 0.8, v["g_pre"], 1e-3)[0]
    got = R.block_norm_bwd(xo, v["y"], v["g_post"], v["gate"], 0.8, v["g_pre"], 1e-3, dxo, dh)
    for k in v:
        if v[k] is not None:
            g, m = got["d" + k]
            assert torch.allclose(g, differences(lambda z: total(**{k: z}), v[k]), atol=1e-7), k
            assert bool((m >= g.abs() - 1e-12).all()), k


def test_lora_gradient():
    v = {"a": rnd(3, 2, 5), "b": rnd(3, 4, 2, seed=1), "x": rnd(6, 5, seed=2)}
    scale, ranks, ids = rnd(3, seed=8), torch.tensor([2, 1, 2]), torch.tensor([0, 1, -1, 1, 3, 0])
    dy, dx = rnd(6, 4, seed=9), rnd(6, 5, seed=10)

    def total(**k):
        u = {**v, **k}
        return (R.lora(u["a"], u["b"], scale, ranks, u["x"], ids, None)[0] * dy).sum()

    low = R.lora(v["a"], v["b"], scale, ranks, v["x"], ids, None)[1]
    got = R.lora_bwd(v["a"], v["b"], scale, ranks, v["x"], low, dy, ids, dx)
    for k, n in (("a", "da"), ("b", "db"), ("x", "out")):
        want = differences(lambda z: total(**{k: z}), v[k]) + (dx if k == "x" else 0)
        assert torch.allclose(got[n][0], want, atol=1e-8), k
