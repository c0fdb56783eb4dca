"""The plain forms of the MXFP4 feed-forward operators: packing against the library's, gradients against differences."""
import numpy as np
import pytest
import torch

import mx_ref as M


def test_pack_is_the_librarys():
    from paper_2608_08910_amd import tq
    g = torch.Generator().manual_seed(1)
    c, _ = M.random_matrix(5, 512, g)
    assert np.array_equal(tq.tq_mx_pack_host(c.numpy()).reshape(-1), M.pack(c).numpy().reshape(-1))
    assert torch.equal(M.unpack(M.pack(c)), c)


def test_quantize_is_nearest():
    g = torch.Generator().manual_seed(2)
    x = torch.randn(7, 256, generator=g, dtype=torch.float64) * torch.exp(3 * torch.randn(7, 1, generator=g, dtype=torch.float64))
    for noclip in (False, True):
        c, s = M.quantize(x, noclip)
        v, b, top = M.values(c, s).reshape(-1, 32), x.reshape(-1, 32), x.reshape(-1, 32).abs().amax(dim=1)
        scale = 2.0 ** (s.reshape(-1).double() - 127)
        # the scale's definition by inequalities
        if noclip:
            assert bool(((top <= 6 * scale) & (top > 3 * scale)).all())
        else:
            assert bool(((top >= 4 * scale) & (top < 8 * scale)).all())
        inside = b.abs() <= 6 * scale[:, None]
        # no representable value is nearer
        grid = torch.cat([-M.E2M1, M.E2M1]) * scale[:, None]
        near = (b[:, :, None] - grid[:, None, :]).abs().amin(dim=2)
        assert bool((((v - b).abs() <= near) | ~inside).all())
        assert torch.equal(v[~inside].abs(), (6 * scale[:, None]).expand_as(v)[~inside])


@pytest.mark.parametrize("kind", [M.SILU, M.GELU])
def test_gradients_against_differences(kind):
    g = torch.Generator().manual_seed(3)
    rnd = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    x, wg, wu, ga, ua, dh = rnd(3, 8), rnd(5, 8), rnd(5, 8), rnd(3, 5), rnd(3, 5), rnd(3, 5)
    _, gp, up = M.gated(kind, x, wg, wu, ga, ua)
    dg, du = M.gated_bwd(kind, gp, up, dh)
    dx = dg @ wg + du @ wu
    h = 1e-6

    def loss(x, ga, ua):
        return (M.gated(kind, x, wg, wu, ga, ua)[0] * dh).sum()
    for name, base, grad in (("x", x, dx), ("ga", ga, dg), ("ua", ua, du)):
        for i in range(base.numel()):
            e = torch.zeros_like(base).reshape(-1)
            e[i] = h
            e = e.reshape(base.shape)
            a = {"x": x, "ga": ga, "ua": ua}
            num = (loss(**{**a, name: base + e}) - loss(**{**a, name: base - e})) / (2 * h)
            assert abs(float(num - grad.reshape(-1)[i])) < 1e-7 * (1 + abs(float(num))), (name, i)
