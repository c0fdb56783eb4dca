"""Router, balance loss and their gradients on the GPU against the plain 64-bit forms."""
import math

import pytest
import torch

import ops_ref as R
from gpu_util import announce, device

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def tq():
    device()
    from paper_2608_08910_amd import tq as _tq
    return _tq


def make(t, e, dtype, seed, kind="plain"):
    """(logits in dtype on the CPU, mask or None). Values stay within +-12 unless the kind says otherwise."""
    g = torch.Generator().manual_seed(1000 * seed + 7 * t + e)
    l = (torch.randn(t, e, generator=g) * 2).clamp(-12, 12)
    mask = None
    if kind == "masked":
        mask = (torch.rand(t, generator=g) < 0.6).to(torch.uint8)
        mask[0] = 0
        l[mask == 0] = math.nan  # a padded row may hold anything
    elif kind == "allmasked":
        mask = torch.zeros(t, dtype=torch.uint8)
    elif kind == "closed":
        l = l.masked_fill(torch.rand(t, e, generator=g) < 0.5, -math.inf)
        l[:, e // 2] = -math.inf
        l[t // 2] = -math.inf
        l[t - 1, 1:] = -math.inf
    elif kind == "ties":
        l = torch.round(l)
        l = torch.where((l == 0) & (torch.rand(t, e, generator=g) < 0.5), -0.0, l)
    elif kind == "lowest":
        l = torch.where(torch.rand(t, e, generator=g) < 0.9, torch.finfo(dtype).min, l)
        l[t // 2] = torch.finfo(dtype).min
    return l.to(dtype), mask


def probs_tol(l, e):
    """Relative bound of a probability. The argument of the exponential is rounded once (half a step of
    up to the span, an absolute error that the exponential makes relative), exp itself and its own
    argument reduction stay within 4 half steps, the sum's additions (e / 64 in a lane, 6 in the
    wave) and the division add one half step each; the sum carries its terms' bound once more."""
    fin = l[torch.isfinite(l.float()) & (l.float() > -1e4)]
    span = float(fin.max() - fin.min()) if fin.numel() else 0.0
    return (2 * (span + 4) + e / 64 + 10) * R.U


def run(tq, l, mask, topk, renorm, alpha=0.02, off=0):
    g = R.Guards()
    t, e = l.shape
    o = dict(idx=g.new((t, topk), torch.int32), w=g.new((t, topk), off=1), counts=g.new((e,), torch.int32), p_mean=g.new((e,)),
             coef=g.new((e,)), loss=g.new((1,)))
    ld = R.offset(l, off)
    md = None if mask is None else mask.cuda()
    tq.tq_route_balance(ld, o["idx"], o["w"], o["counts"], o["p_mean"], o["coef"], o["loss"], tq.route_workspace(t, e), alpha,
                        token_mask=md, flags=tq.TQ_ROUTE_RENORM if renorm else 0)
    i2, w2 = g.new((t, topk), torch.int32), g.new((t, topk))
    tq.tq_route(ld, i2, w2, token_mask=md, flags=tq.TQ_ROUTE_RENORM if renorm else 0)
    torch.cuda.synchronize()
    g.check()
    assert torch.equal(i2, o["idx"])
    return o, w2, ld, md


CASES = [(1, 1, 1, F32, "plain"), (1, 256, 8, F32, "plain"), (3, 2, 2, BF16, "plain"), (5, 7, 3, F16, "ties"),
         (2, 60, 60, F32, "closed"), (33, 64, 6, BF16, "ties"), (17, 65, 64, F32, "plain"), (64, 129, 5, F16, "closed"),
         (9, 256, 8, F16, "lowest"), (16, 256, 8, BF16, "masked"), (4, 256, 1, F32, "allmasked"), (130, 256, 8, F32, "closed"),
         (31, 300, 9, BF16, "lowest"), (12, 512, 16, F32, "ties"), (7, 1000, 10, BF16, "plain"), (5, 1024, 64, F16, "masked"),
         (3, 1025, 8, F32, "closed"), (2, 4096, 64, F32, "ties"), (6, 4095, 7, BF16, "masked"), (2051, 96, 4, BF16, "masked")]


@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("t,e,topk,dtype,kind", CASES)
def test_route_balance_and_gradient(tq, t, e, topk, dtype, kind, renorm):
    announce(f"route t={t} E={e} topk={topk} {dtype} {kind} renorm={renorm}")
    l, mask = make(t, e, dtype, 1, kind)
    idx, w, p = R.route(l.double(), topk, renorm, mask)
    counts, mean, coef, loss = R.balance(idx, p, topk, 0.02, mask)
    o, w2, ld, md = run(tq, l, mask, topk, renorm, off=(t + topk) % 4)
    tol = probs_tol(l, e)
    assert torch.equal(o["idx"].cpu().long(), idx)
    R.close(o["w"], w, tol * w + R.TINY[F32], "w")
    R.close(w2, w, tol * w + R.TINY[F32], "w (tq_route)")
    assert torch.equal(o["counts"].cpu().long(), counts)
    # a workgroup's sum adds a wave's tokens one by one and its four waves
    per = math.ceil(t / (4 * min(512, max(1, math.ceil(t / 16))))) + 6
    R.close(o["p_mean"], mean, (tol + per * R.U) * mean + R.TINY[F32], "p_mean")
    R.close(o["coef"], coef, 2 * R.U * coef + R.TINY[F32], "coef")
    R.close(o["loss"], loss, (tol + (per + 2) * R.U) * loss + R.TINY[F32], "loss")

    g = torch.Generator().manual_seed(t + e)
    dw = torch.randn(t, topk, generator=g)
    dloss = torch.tensor([0.7])
    for use_w, use_b in ((True, True), (True, False), (False, True)):
        ref, mag = R.route_bwd(idx, w, p, renorm, dw.double() if use_w else None, coef if use_b else None, float(dloss))
        gd = R.Guards()
        dl = gd.new((t, e), dtype, off=1)
        tq.tq_route_bwd(ld, o["idx"], o["w"], dl, dw=dw.cuda().masked_fill(o["idx"] < 0, math.nan) if use_w else None,
                        coef=o["coef"] if use_b else None, dloss=dloss.cuda() if use_b else None, token_mask=md,
                        flags=tq.TQ_ROUTE_RENORM if renorm else 0)
        torch.cuda.synchronize()
        gd.check()
        # every term has p (or w) once, its sums twice, and up to e / 64 + 16 additions
        R.close(dl, ref, (3 * tol + (e / 64 + 24) * R.U) * mag + R.HALF[dtype] * ref.abs() + R.TINY[dtype], f"dlogits {use_w} {use_b}")


def test_gradient_in_place_and_equal_bits(tq):
    t, e, topk = 700, 256, 8
    l, mask = make(t, e, F32, 5)
    o, _, ld, md = run(tq, l, mask, topk, True)
    p, _, _, _ = run(tq, l, mask, topk, True)
    assert all(torch.equal(o[k], p[k]) for k in o)
    dw, dloss = torch.randn(t, topk, device="cuda"), torch.ones(1, device="cuda")
    a = torch.empty_like(ld)
    tq.tq_route_bwd(ld, o["idx"], o["w"], a, dw=dw, coef=o["coef"], dloss=dloss, flags=1)
    tq.tq_route_bwd(ld, o["idx"], o["w"], ld, dw=dw, coef=o["coef"], dloss=dloss, flags=1)
    assert torch.equal(a, ld)


def test_a_nan_or_infinite_logit_shows(tq):
    l, _ = make(4, 100, F32, 2)
    l[1, 3], l[2, 9] = math.nan, math.inf
    o, w2, _, _ = run(tq, l, None, 5, False)
    for row in (1, 2):
        assert bool(torch.isnan(o["w"][row]).all()) and bool(torch.isnan(w2[row]).all())
        ids = o["idx"][row].tolist()
        assert len(set(ids)) == 5 and min(ids) >= 0 and max(ids) < 100
    assert bool(torch.isfinite(o["w"][[0, 3]]).all())


@pytest.mark.parametrize("t,e,topk,kind", [(40, 64, 8, "ties"), (33, 100, 12, "closed"), (21, 256, 16, "ties"), (9, 512, 32, "lowest"),
                                           (70, 16, 16, "ties"), (12, 1030, 8, "ties"), (8, 8, 8, "masked"), (5, 2047, 20, "closed")])
def test_many_slots(tq, t, e, topk, kind):
    """Equal keys at the last slot, fewer experts than slots, all of them chosen."""
    announce(f"many slots t={t} e={e} topk={topk} {kind}")
    l, mask = make(t, e, F32, 9, kind)
    idx, w, _ = R.route(l.double(), topk, True, mask)
    o, w2, _, _ = run(tq, l, mask, topk, True)
    assert torch.equal(o["idx"].cpu().long(), idx)
    R.close(o["w"], w, 2 * probs_tol(l, e) * w + R.TINY[F32], "w")
    assert torch.equal(o["w"], w2)


def test_a_nan_among_many_slots(tq):
    l, _ = make(3, 100, F32, 2)
    l[1, [3, 77]] = math.nan
    o, _, _, _ = run(tq, l, None, 9, True)
    ids = o["idx"].cpu()
    assert ids[1, :2].tolist() == [3, 77] and all(len(set(r)) == 9 for r in ids.tolist()) and int(ids.min()) >= 0
    assert bool(torch.isnan(o["w"][1]).all()) and bool(torch.isfinite(o["w"][[0, 2]]).all())


def test_no_tokens(tq):
    e = 20
    g = R.Guards()
    c, m, f, s = g.new((e,), torch.int32), g.new((e,)), g.new((e,)), g.new((1,))
    z = lambda *sh, dtype=F32: torch.empty(sh, dtype=dtype, device="cuda")  # noqa: E731
    tq.tq_route(z(0, e), z(0, 3, dtype=torch.int32), z(0, 3))
    tq.tq_route_bwd(z(0, e), z(0, 3, dtype=torch.int32), z(0, 3), z(0, e), dw=z(0, 3))
    tq.tq_route_balance(z(0, e), z(0, 3, dtype=torch.int32), z(0, 3), c, m, f, s, tq.route_workspace(0, e), 1.0)
    torch.cuda.synchronize()
    g.check()
    assert not bool(c.any()) and not bool(m.any()) and not bool(f.any()) and float(s) == 0.0


@pytest.mark.parametrize("t,topk,h", [(1, 1, 256), (1, 8, 7168), (3, 7, 512), (33, 8, 1024), (5, 64, 256), (300, 6, 4096), (2, 3, 16384)])
def test_weight_grad(tq, t, topk, h):
    announce(f"weight_grad t={t} topk={topk} h={h}")
    g = torch.Generator().manual_seed(t * topk + h)
    yd, dout = torch.randn(t * topk, h, generator=g), torch.randn(t, h, generator=g)
    idx = torch.randint(0, 16, (t, topk), generator=g, dtype=torch.int32)
    idx[torch.rand(t, topk, generator=g) < 0.2] = -1
    idx[torch.rand(t, topk, generator=g) < 0.1] = 16
    off = (idx < 0) | (idx >= 16)
    yd[off.reshape(-1)] = math.nan  # never written by the layer's call
    prod = (yd.double().view(t, topk, h) * dout.double()[:, None]).masked_fill(off[..., None], 0.0)
    gd = R.Guards()
    dw = gd.new((t, topk))
    tq.tq_moe_weight_grad(yd.cuda(), dout.cuda(), idx.cuda(), dw, 16)
    torch.cuda.synchronize()
    gd.check()
    # a lane adds h / 64 products one after the other, then 8 additions join the lanes
    R.close(dw, prod.sum(2), (h / 64 + 10) * R.U * prod.abs().sum(2), "dw")


@pytest.mark.parametrize("t,e,topk,dtype,kind", [(40, 64, 33, BF16, "ties"), (33, 100, 31, F16, "closed"), (21, 256, 32, BF16, "ties"), (9, 512, 20, F16, "lowest"),
                                                 (5, 1024, 63, BF16, "closed"), (4, 2000, 64, F16, "ties"), (3, 4096, 12, BF16, "ties"), (6, 4096, 64, F16, "lowest")])
def test_sixteen_bit_logits(tq, t, e, topk, dtype, kind):
    """Keys that carry their expert: equal values, the type's lowest, the highest ids."""
    announce(f"tagged t={t} e={e} topk={topk} {dtype} {kind}")
    l, mask = make(t, e, dtype, 12, kind)
    l[0, e - 1] = 12.0  # the last id is among the chosen
    if dtype == F16:
        l[1, :4] = torch.tensor([5.9604644775390625e-08, -5.9604644775390625e-08, 0.0, -0.0]).to(F16)  # the least subnormals
    idx, w, p = R.route(l.double(), topk, False, mask)
    o, w2, _, _ = run(tq, l, mask, topk, False)
    assert torch.equal(o["idx"].cpu().long(), idx)
    R.close(o["w"], w, probs_tol(l, e) * w + R.TINY[F32], "w")
    R.close(w2, w, probs_tol(l, e) * w + R.TINY[F32], "w")
    counts, mean, _, _ = R.balance(idx, p, topk, 0.02, mask)
    assert torch.equal(o["counts"].cpu().long(), counts.long())
    R.close(o["p_mean"], mean, (probs_tol(l, e) + 8 * R.U) * mean + R.TINY[F32], "p_mean")


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_a_nan_among_sixteen_bit_logits(tq, dtype):
    l, _ = make(3, 300, dtype, 2)
    l[1, [3, 277]] = math.nan
    l[2, 200] = math.inf
    o, w2, _, _ = run(tq, l, None, 9, False)
    ids = o["idx"].cpu()
    assert ids[1, :2].tolist() == [3, 277] and ids[2, 0] == 200 and all(len(set(r)) == 9 for r in ids.tolist())
    for v in (o["w"], w2):
        assert bool(torch.isnan(v[1:]).all()) and bool(torch.isfinite(v[0]).all())


@pytest.mark.parametrize("t,e,topk,dtype", [(1, 1, 1, F32), (37, 64, 8, BF16), (50, 129, 5, F32), (33, 256, 8, F16), (21, 1001, 9, BF16),
                                            (9, 4096, 64, F32), (6, 4095, 7, F16)])
@pytest.mark.parametrize("renorm", [0, 1])
def test_gradient_in_place_of_every_width(tq, t, e, topk, dtype, renorm):
    announce(f"route gradient in place t={t} E={e} topk={topk} {dtype} renorm={renorm}")
    l, mask = make(t, e, dtype, 15, "masked" if t > 1 else "plain")
    o, _, ld, md = run(tq, l, mask, topk, bool(renorm), off=1)
    g = torch.Generator(device="cuda").manual_seed(e)
    kw = dict(dw=torch.randn(t, topk, device="cuda", generator=g), coef=o["coef"], dloss=torch.ones(1, device="cuda"), token_mask=md, flags=renorm)
    gd = R.Guards()
    a, b = gd.new((t, e), dtype, off=3), gd.new((t, e), dtype, off=1)
    b.copy_(ld)
    tq.tq_route_bwd(ld, o["idx"], o["w"], a, **kw)
    tq.tq_route_bwd(b, o["idx"], o["w"], b, **kw)
    torch.cuda.synchronize()
    gd.check()
    assert torch.equal(a, b) and bool(a.any()) == (e > 1)


@pytest.mark.parametrize("t,topk,h", [(64, 8, 1024), (73, 7, 1024), (27, 19, 256), (128, 8, 768), (205, 5, 256)])
def test_weight_grad_about_the_shared_slots(tq, t, topk, h):
    """511 to 1025 slots: on both sides of where the waves of a workgroup stop sharing one."""
    test_weight_grad(tq, t, topk, h)
