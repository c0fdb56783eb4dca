"""What the MXFP4 feed-forward operators keep of their operands' bits: bounds by the values themselves, not by sums of magnitudes."""
import math

import pytest
import torch

import mx_plan as P
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
    four roundings in the cubic term, one in the sum, one and its constant's outside); e = exp(-a) by d = 7 a (SiLU: 0) and 2 of the exponential; q = e / (1 + e)
    by p d + 3, p = 1 - q by q / p times that and 1; a' by 7; the second term by those of p, q and a' and 3; the sum, SiLU's last product and dg's two
    products by 1 each. (q from 1 - p is off by up to U, not relative to q: at z = 5 GELU's z a' makes 35 U of it, where the bound is below 7.)"""
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
    off_q = p * d + 3
    off_p = q / p * off_q + 1
    rel = (off_p + share * (off_q + 7 + 3) + 4) * R.U * 1.01  # (1.01: products of these errors)
    ref, _ = M.gated_bwd(kind, x, u.double(), dh.double())
    R.close(dg, ref, rel * ref.abs() + R.TINY[F32], "dg")


@pytest.mark.parametrize("kind", [M.SILU, M.GELU])
def test_activation_of_large_arguments(tq, kind):
    """du = act(z), z > 0, dh = 1, in fp32: p = 1 - q lies between 1/2 and 1, where half a step is 2^-25, and is off by that and by q's own
    error (above); z p and du by half a step of theirs. (1 / (1 + e) is off by half a step of 1 + e as well, 2^-24.)"""
    n, k, t = 1024, 256, 64
    g = torch.Generator().manual_seed(22)
    w = matrix(tq, *M.random_matrix(n, k, g))
    z = 1 + torch.rand(t, n, generator=g) * (19 if kind == M.SILU else 4.5)
    one = torch.ones(t, n, device="cuda")
    dg, du = torch.empty(t, n, device="cuda"), torch.empty(t, n, device="cuda")
    announce(f"activation act={kind}")
    tq.tq_gated_mx_bwd(w, w, z.cuda(), one, one, dg, du, None, None, act=kind)
    torch.cuda.synchronize()
    x = z.double()
    a = x if kind == M.SILU else 2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)
    p, q = torch.sigmoid(a), torch.sigmoid(-a)
    d = (0 if kind == M.SILU else 7 * a) + 2
    ref = M.act(kind, x)
    half = torch.exp2(torch.floor(torch.log2(ref)) - 24)
    R.close(du, ref, x * (2.0 ** -25 + q * (p * d + 3) * R.U * 1.01) + half * (1 + 2.0 ** -20), "du")


def last_bits(shape, dt, g):
    """Values of 1 to 2, signs mixed, whose last bit is set: nearly all of fp32's take three bfloat16 parts, fp16's two."""
    digits = {F32: 24, BF16: 8, F16: 11}[dt]
    v = (torch.randint(1 << (digits - 1), 1 << digits, shape, generator=g) | 1).double() * 2.0 ** (1 - digits)
    return torch.where(torch.rand(shape, generator=g) < 0.5, -v, v).to(dt)


def check_products(dx, value, w, what):
    """dx against one value of dy a row (float64) times its row w of weights: exact where fp32 holds the product (bfloat16 and fp16 values, and
    any times a power of two), rounded once to dx's type; else fp32's lowest parts' sum is exact and one addition is rounded or cut off."""
    ref = value[:, None] * w
    exact = ref.to(dx.dtype) if dx.dtype != F32 else ref.float()
    power = torch.frexp(w)[0].abs() == 0.5
    if dx.dtype != F32:
        power = torch.ones_like(power)
    same = (dx == exact) | ~(power | (w == 0))
    near = (dx.double() - ref).abs() <= 2.0 ** -23 * ref.abs() if dx.dtype == F32 else torch.ones_like(same)
    assert bool((same & near).all()), (what, int((~same).sum()), int((~near).sum()))


@pytest.mark.parametrize("n,k,t", P.SIZES)
def test_gradients_of_single_values(tq, n, k, t):
    """dy with one value a row: dx is its product with one row of weights, which shows a lost part of a value, a lost or doubled step, and a
    sum of the wrong rows, in every way that the gradients take."""
    g = torch.Generator().manual_seed(n + t)
    (cg, sg), (cu, su) = M.random_matrix(n, k, g), M.random_matrix(n, k, g)
    wg, wu = M.values(cg, sg).cuda(), M.values(cu, su).cuda()
    dwg, dwu = matrix(tq, cg, sg), matrix(tq, cu, su)
    at = torch.cat([torch.randperm(n, generator=g) for _ in range(-(-t // n))])[:t]
    at[0], rows = n - 1, torch.arange(t)
    for ty, dt in enumerate(TYPES):
        v = last_bits((t,), dt, g)
        announce(f"single values n={n} k={k} t={t} {dt} {P.way(P.plan(n, k, t, 1, ty))} {P.way(P.plan(n, k, t, 2, ty))}")
        dy = torch.zeros(t, n, dtype=dt)
        dy[rows, at] = v
        for off in (0, 1):
            gd = R.Guards()
            dx = gd.new((t, k), dt, off=off)
            tq.tq_gemm_mx_bwd(dwg, R.offset(dy, off), dx, tq.gemm_mx_bwd_workspace(dwg, t, dt).fill_(255))
            torch.cuda.synchronize()
            gd.check()
            check_products(dx, v.double().cuda(), wg[at.cuda()], ("dx", dt, off))
        # both matrices: dg alone where g = 0 and u = 2 (act(0) = 0, act'(0) = 1/2: dg = dh), du alone where u = 0
        gate = torch.rand(t, generator=g) < 0.5
        gp, up = torch.full((t, n), 1.5, dtype=dt), torch.zeros(t, n, dtype=dt)
        gp[gate], up[gate] = 0.0, 2.0
        for off in (0, 1):
            gd = R.Guards()
            dg, du, dx = gd.new((t, n), dt, off=off), gd.new((t, n), dt, off=off), gd.new((t, k), dt)
            tq.tq_gated_mx_bwd(dwg, dwu, gp.cuda(), up.cuda(), dy.cuda(), dg, du, dx, tq.gated_mx_bwd_workspace(dwg, dwu, t, dt).fill_(255),
                               act=(M.SILU, M.GELU)[off])
            torch.cuda.synchronize()
            gd.check()
            assert torch.equal(dg.cpu(), torch.where(gate[:, None], dy, 0)) and not bool(du.cpu()[gate].any())
            w = torch.where(gate[:, None].cuda(), wg[at.cuda()], wu[at.cuda()])
            value = torch.where(gate.cuda(), dg[rows, at], du[rows, at])
            assert bool((value != 0).all()) and int((du != 0).sum()) == int((~gate).sum())
            check_products(dx, value.double(), w, ("gated dx", dt, off))
