"""What the MXFP4 feed-forward operators keep of their operands' bits: bounds by the values themselves, not by sums of magnitudes."""
import math

import pytest
import torch

import mx_ref as M
import ops_ref as R
from gpu_util import announce
from test_gpu_mx_block import TYPES, matrix, tq  # noqa: F401  (tq: the module's fixture)

pytestmark = pytest.mark.gpu
F32, BF16, F16 = TYPES


@pytest.mark.parametrize("kind", [M.SILU, M.GELU])
def test_derivative_of_large_arguments(tq, kind):
    """dg = dh u act'(z), z >= 0, in fp32, where act' = p + z p q a' (q = 1 - p, a' = 1 for SiLU) is a sum of positive terms, so that its
    relative error is that of its terms, weighted by their shares. In half steps U of fp32: GELU's argument a is off by at most 7 (one and
    four roundings in the cubic term, one in the sum, one and its constant's outside); e = exp(-a) by d = 7 a (SiLU: 0) and 2 of the exponential; p = 1 / (1 + e)
    by q d + 2, q = e p by d + 3; a' by 7; the second term by those of p, q and a' and 3; the sum, SiLU's last product and dg's two products by 1 each.
    (1 - p instead of e p is off by up to U, not relative to q: at z = 5 GELU's z a' makes 35 U of it, where the bound is below 7.)"""
    n, k, t = 1024, 256, 64
    g = torch.Generator().manual_seed(21)
    w = matrix(tq, *M.random_matrix(n, k, g))
    z = (torch.rand(t, n, generator=g) * torch.linspace(1, 30, t)[:, None])
    u, dh = (torch.randn(t, n, generator=g) for _ in range(2))
    dg, du = torch.empty(t, n, device="cuda"), torch.empty(t, n, device="cuda")
    announce(f"derivative act={kind}")
    tq.tq_gated_mx_bwd(w, w, z.cuda(), u.cuda(), dh.cuda(), dg, du, None, None, act=kind)
    torch.cuda.synchronize()
    x, two_a = z.double(), 2 * math.sqrt(2 / math.pi)
    a, da = (x, torch.ones_like(x)) if kind == M.SILU else (two_a * (x + 0.044715 * x ** 3), two_a * (1 + 3 * 0.044715 * x * x))
    p, q = torch.sigmoid(a), torch.sigmoid(-a)
    d = (0 if kind == M.SILU else 7 * a) + 2
    second = x * p * q * da
    share = second / (p + second)
    rel = (q * d + 2 + share * (d + 3 + 7 + 3) + 4) * R.U * 1.01  # (1.01: products of these errors)
    ref, _ = M.gated_bwd(kind, x, u.double(), dh.double())
    R.close(dg, ref, rel * ref.abs() + R.TINY[F32], "dg")
