"""The MXFP4 feed-forward operators as a training batch uses them, and with codes, rows and gradients past 4 GB."""
import pytest
import torch

import mx_ref as M
import ops_ref as R
from gpu_util import announce
from test_gpu_mx_block import TYPES, act_error, matrix, product_bound, tq  # noqa: F401  (tq: the module's fixture)
from test_gpu_mx_precision import check_products, last_bits

pytestmark = pytest.mark.gpu
F32, BF16, F16 = TYPES


# tiles of 64 x 64, of 128 x 128 in four stages and in two, of 256 x 256; with edges in both directions
@pytest.mark.parametrize("n,k,t", [(1000, 768, 300), (1100, 512, 1000), (2050, 512, 1300), (2050, 768, 2101)])
@pytest.mark.parametrize("kind", [M.SILU, M.GELU])
def test_gated_with_everything(tq, n, k, t, kind):
    """Each type with adapters' parts on both projections, on one or none, the pre-activations kept or not."""
    g = torch.Generator().manual_seed(n + t)
    (cg, sg), (cu, su), (cx, sx) = M.random_matrix(n, k, g), M.random_matrix(n, k, g), M.random_matrix(t, k, g)
    wg, wu, x = M.values(cg, sg).cuda(), M.values(cu, su).cuda(), M.values(cx, sx).cuda()
    dg, du, dx = matrix(tq, cg, sg), matrix(tq, cu, su), matrix(tq, cx, sx)
    ga, ua = (torch.randn(t, n, generator=g).cuda() for _ in range(2))
    pg, pu = x @ wg.t().contiguous(), x @ wu.t().contiguous()
    bg, bu = (product_bound(k // 64, x.abs() @ w.abs().t().contiguous()) for w in (wg, wu))
    for dt in TYPES:
        for add in (2, 1, 0):
            for save in (True, False):
                announce(f"gated with everything n={n} k={k} t={t} {dt} act={kind} add={add} save={save}")
                gd = R.Guards()
                h, go, uo = (gd.new((t, n), dt) for _ in range(3))
                if not save:
                    go = uo = None
                tq.tq_gated_mx(dg, du, dx, h, act=kind, g_add=ga if add else None, u_add=ua if add == 2 else None, g=go, u=uo)
                torch.cuda.synchronize()
                gd.check()
                gp, up = (pg + ga if add else pg), (pu + ua if add == 2 else pu)
                # (the sums' bound, and the addition's rounding)
                eg, eu = bg + R.U * (gp.abs() + bg), bu + R.U * (up.abs() + bu)

                def off(got, ref, e):
                    return bool(((got.double() - ref).abs() <= e + R.HALF[dt] * (ref.abs() + e) + R.TINY[dt]).all())
                if save:
                    assert off(go, gp, eg) and off(uo, up, eu)
                # (|act'| < 1.13; act and the product are rounded once each)
                a = M.act(kind, gp)
                ea = 1.2 * eg + act_error(kind, gp)
                eh = ea * (up.abs() + eu) + a.abs() * eu + 2 * R.U * (a * up).abs()
                assert off(h, a * up, eh)


# ---- past 4 GB: rows on both sides of 2^32 bytes of codes, and the last ones ------------------------

K = 16384
ROWS = 600000  # 8 KB of codes each
AT = [0, 1, 300001, (1 << 32) // (K // 2) - 1, (1 << 32) // (K // 2), ROWS - 2, ROWS - 1]


@pytest.fixture(scope="module")
def far(tq):
    """(a matrix of 4.9 GB of codes, its rows AT in 64 bits)."""
    g = torch.Generator(device="cuda").manual_seed(5)
    m = tq.TqMatrixMx.empty(ROWS, K)
    for a in range(0, ROWS, 100000):
        m.codes[a:a + 100000] = torch.randint(0, 256, m.codes[a:a + 100000].shape, generator=g, device="cuda", dtype=torch.uint8)
        m.scales[a:a + 100000] = 118 + torch.randint(0, 8, m.scales[a:a + 100000].shape, generator=g, device="cuda", dtype=torch.uint8)
    yield m, M.values(M.unpack(m.codes[AT].cpu()), m.scales[AT].cpu())
    del m
    torch.cuda.empty_cache()


@pytest.mark.parametrize("t", [1, 30, 200])
def test_far_weights(tq, far, t):
    w, rows = far
    g = torch.Generator().manual_seed(t)
    cx, sx = M.random_matrix(t, K, g)
    x = M.values(cx, sx)
    announce(f"far weights t={t}")
    y = torch.empty(t, ROWS, dtype=BF16, device="cuda")
    tq.tq_gemm_mx(w, matrix(tq, cx, sx), y)
    ref, b = x @ rows.t(), product_bound(K // 64, x.abs() @ rows.abs().t())
    R.close(y[:, AT], ref, b + R.HALF[BF16] * (ref.abs() + b), "y")
    h, go, uo = (torch.empty(t, ROWS, dtype=F32, device="cuda") for _ in range(3))
    tq.tq_gated_mx(w, w, matrix(tq, cx, sx), h, g=go, u=uo)
    R.close(go[:, AT], ref, b, "g")
    assert torch.equal(go, uo)


@pytest.mark.parametrize("t", [5, 70])
def test_far_weights_gradient(tq, far, t):
    w, rows = far
    g = torch.Generator().manual_seed(t)
    at = torch.arange(t) % len(AT)
    for dt in TYPES:
        announce(f"far weights' gradient t={t} {dt}")
        v = last_bits((t,), dt, g)
        dy = torch.zeros(t, ROWS, dtype=dt, device="cuda")
        dy[torch.arange(t), torch.tensor(AT)[at]] = v.cuda()
        dx = torch.empty(t, K, dtype=dt, device="cuda")
        tq.tq_gemm_mx_bwd(w, dy, dx, tq.gemm_mx_bwd_workspace(w, t, dt).fill_(255))
        check_products(dx.cpu(), v.double(), rows[at], dt)


def test_far_rows(tq, far):
    x, rows = far
    g = torch.Generator().manual_seed(6)
    (cg, sg), (cu, su) = M.random_matrix(20, K, g), M.random_matrix(20, K, g)
    wg, wu = M.values(cg, sg), M.values(cu, su)
    announce("far rows")
    h, go, uo = (torch.empty(ROWS, 20, dtype=F32, device="cuda") for _ in range(3))
    tq.tq_gated_mx(matrix(tq, cg, sg), matrix(tq, cu, su), x, h, g=go, u=uo)
    for o, w in ((go, wg), (uo, wu)):
        R.close(o[AT], rows @ w.t(), product_bound(K // 64, rows.abs() @ w.abs().t()), "far rows")
    y = torch.empty(ROWS, 20, dtype=F32, device="cuda")
    tq.tq_gemm_mx(matrix(tq, cg, sg), x, y)
    R.close(y[AT], rows @ wg.t(), product_bound(K // 64, rows.abs() @ wg.abs().t()), "far rows")


def test_far_quantization(tq):
    """Rows of 2^32 elements, in place too, against those of a few rows by themselves."""
    t = 300000
    at = torch.tensor([0, 1, 131071, 131072, 262143, 262144, t - 1], device="cuda")
    x = torch.empty(t, K, dtype=BF16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(7))
    x[at] *= torch.linspace(0.5, 3, len(at), device="cuda").to(BF16)[:, None]
    few = x[at].contiguous()
    c, s = M.quantize(few.cpu().double())
    announce("far quantization")
    m = tq.TqMatrixMx.empty(t, K)
    tq.tq_quantize_mx(x, m, values=x)
    torch.cuda.synchronize()
    assert torch.equal(M.unpack(m.codes[at].cpu()), c) and torch.equal(m.scales[at].cpu(), s)
    assert torch.equal(x[at].cpu().double(), M.values(c, s))
    del x, m
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dt", TYPES)
def test_far_input_gradient(tq, dt):
    """dx past 2^32 elements, by one value of dy a row."""
    n, t = 24, 300000
    g = torch.Generator().manual_seed(8)
    cw, sw = M.random_matrix(n, K, g)
    w, wv = matrix(tq, cw, sw), M.values(cw, sw)
    v, at = last_bits((t,), dt, g), torch.arange(t) % n
    dy = torch.zeros(t, n, dtype=dt, device="cuda")
    dy[torch.arange(t), at] = v.cuda()
    announce(f"far dx {dt}")
    dx = torch.empty(t, K, dtype=dt, device="cuda")
    tq.tq_gemm_mx_bwd(w, dy, dx, tq.gemm_mx_bwd_workspace(w, t, dt))
    rows = torch.tensor([0, 1, 131071, 131072, 262143, 262144, t - 2, t - 1])
    check_products(dx[rows.cuda()].cpu(), v[rows].double(), wv[at[rows]], dt)
    del dx
    torch.cuda.empty_cache()


@pytest.mark.parametrize("n", [2304, 2305])
def test_far_gated_gradient(tq, n):
    """The most rows that a call takes, with dg, du and (n odd) dy's copies past 2^31 elements; dh is zero but in a few rows."""
    t, k, dt = 1 << 20, 256, BF16
    g = torch.Generator().manual_seed(n)
    (cg, sg), (cu, su) = M.random_matrix(n, k, g), M.random_matrix(n, k, g)
    dwg, dwu, wg = matrix(tq, cg, sg), matrix(tq, cu, su), M.values(cg, sg)
    rows = torch.tensor([0, 5, (1 << 31) // n, (1 << 31) // n + 1, t - 2, t - 1])
    v, at = last_bits((len(rows),), dt, g), torch.tensor([n - 1, 0, n // 2, n - 1, 3, n - 1])
    gp, up = torch.zeros(t, n, dtype=dt, device="cuda"), torch.full((t, n), 2.0, dtype=dt, device="cuda")
    dh = torch.zeros(t, n, dtype=dt, device="cuda")
    dh[rows.cuda(), at.cuda()] = v.cuda()
    announce(f"far gated gradient n={n}")
    dg, du, dx = torch.empty_like(dh), torch.empty_like(dh), torch.empty(t, k, dtype=dt, device="cuda")
    tq.tq_gated_mx_bwd(dwg, dwu, gp, up, dh, dg, du, dx, tq.gated_mx_bwd_workspace(dwg, dwu, t, dt))
    torch.cuda.synchronize()
    assert torch.equal(dg, dh) and not bool(du.any())  # (act(0) = 0 and act'(0) = 1/2, u = 2)
    check_products(dx[rows.cuda()].cpu(), v.double(), wg[at], n)
    dx[rows.cuda()] = 0
    assert not bool(dx.any())
    del gp, up, dh, dg, du, dx
    torch.cuda.empty_cache()
