"""What the router, the block norms and the adapters refuse, before any launch (host only: the device
pointers here are made up, so nothing here may reach a launch)."""
import ctypes

import pytest
import torch

from paper_2608_08910_amd import _tqpy as fast
from paper_2608_08910_amd import tq

host_only = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up device pointers; host-only")
L = tq._L
P = 1 << 20  # a made-up, well aligned device address
INV, ALIGN, WS = tq.TQ_ERR_INVALID, tq.TQ_ERR_ALIGN, tq.TQ_ERR_WORKSPACE


def refuse(fn, good, changes):
    """Each change of the good arguments (name -> value) gives its status and a message that names the call.
    (The good call itself is never made.)"""
    for ch, status in changes:
        a = {**good, **ch}
        st = fn(*a.values())
        msg = tq.tq_last_error()
        assert st == status and fn.__name__ in msg, (fn.__name__, ch, st, msg)


@host_only
def test_route_refusals():
    good = dict(logits=P, type=0, t=4, e=16, mask=P, topk=2, flags=0, idx=P, w=P, stream=None)
    common = [(dict(type=3), INV), (dict(type=-1), INV), (dict(t=-1), INV), (dict(t=(1 << 24) + 1), INV), (dict(e=0), INV),
              (dict(e=4097), INV), (dict(topk=0), INV), (dict(topk=17), INV), (dict(topk=65, e=100), INV), (dict(flags=2), INV),
              (dict(logits=0), INV), (dict(idx=0), INV), (dict(w=0), INV), (dict(logits=P + 2), ALIGN), (dict(logits=P + 1, type=1), ALIGN),
              (dict(idx=P + 2), ALIGN), (dict(w=P + 1), ALIGN)]
    refuse(L.tq_route, good, common)
    need = tq.tq_route_workspace_bytes(4, 16)
    bal = {k: v for k, v in good.items() if k not in ("idx", "w", "stream")}
    bal.update(alpha=1.0, idx=P, w=P, counts=P, mean=P, coef=P, loss=P, ws=P, n=need, stream=None)
    refuse(L.tq_route_balance, bal, common + [(dict(counts=0), INV), (dict(mean=0), INV), (dict(coef=0), INV), (dict(loss=0), INV),
                                              (dict(ws=0), INV), (dict(ws=P + 128), ALIGN), (dict(coef=P + 2), ALIGN),
                                              (dict(n=need - 1), WS), (dict(t=0, ws=0), INV)])
    bwd = {k: v for k, v in good.items() if k != "stream"}
    bwd.update(dw=P, coef=P, dloss=P, dl=P, stream=None)
    refuse(L.tq_route_bwd, bwd, common + [(dict(dl=0), INV), (dict(dw=0, coef=0, dloss=0), INV), (dict(coef=0), INV), (dict(dloss=0), INV),
                                          (dict(dl=P + 2), ALIGN), (dict(dw=P + 2), ALIGN)])
    wg = dict(yd=P, dout=P, t=2, h=256, idx=P, topk=2, e=8, dw=P, stream=None)
    refuse(L.tq_moe_weight_grad, wg, [(dict(t=-1), INV), (dict(t=(1 << 20) + 1), INV), (dict(h=0), INV), (dict(h=300), INV),
                                      (dict(h=16640), INV), (dict(topk=0), INV), (dict(topk=65), INV), (dict(e=0), INV), (dict(e=4097), INV),
                                      (dict(yd=0), INV), (dict(dout=0), INV), (dict(idx=0), INV), (dict(dw=0), INV), (dict(yd=P + 4), ALIGN),
                                      (dict(dout=P + 8), ALIGN), (dict(dw=P + 2), ALIGN)])
    for t, e in ((-1, 8), ((1 << 24) + 1, 8), (4, 0), (4, 4097)):
        assert tq.tq_route_workspace_bytes(t, e) == 0
    # no tokens: nothing to do, nothing touched
    assert L.tq_route(*{**good, "t": 0, "logits": 0, "idx": 0, "w": 0}.values()) == 0
    assert L.tq_route_bwd(*{**bwd, "t": 0}.values()) == 0 and L.tq_moe_weight_grad(*{**wg, "t": 0}.values()) == 0


@host_only
def test_block_norm_refusals():
    good = dict(x=P, xt=1, y=P, yt=0, t=4, h=100, g_post=P, gate=P, kind=1, rs=1.0, g_pre=P, eps=1e-6, x_out=P, h_out=P, stream=None)
    common = [(dict(xt=3), INV), (dict(yt=2), INV), (dict(xt=0, yt=1), INV), (dict(t=-1), INV), (dict(t=(1 << 24) + 1), INV),
              (dict(h=0), INV), (dict(h=16385), INV), (dict(kind=3), INV), (dict(kind=-1), INV), (dict(kind=0), INV), (dict(gate=0), INV),
              (dict(eps=0.0), INV), (dict(eps=-1.0), INV), (dict(eps=float("nan")), INV), (dict(eps=2.0), INV), (dict(g_post=P + 2), ALIGN),
              (dict(gate=P + 2), ALIGN), (dict(g_pre=P + 1), ALIGN)]
    refuse(L.tq_block_norm, good, common + [
        (dict(x=0), INV), (dict(y=0), INV), (dict(x_out=0), INV), (dict(h_out=0), INV), (dict(g_pre=0), INV),
        (dict(y=0, x_out=0), INV), (dict(y=0, x_out=0, g_post=0, gate=0, kind=0, h_out=0, g_pre=0), INV),
        (dict(x=P + 1), ALIGN), (dict(y=P + 2), ALIGN), (dict(x_out=P + 1), ALIGN), (dict(h_out=P + 2), ALIGN)])
    need = tq.tq_block_norm_workspace_bytes(4, 100)
    bwd = {k: v for k, v in good.items() if k not in ("x_out", "h_out", "stream")}
    bwd.update(dxo=P, dh=P, dx=P, dy=P, dg_post=P, dgate=P, dg_pre=P, ws=P, n=need, stream=None)
    refuse(L.tq_block_norm_bwd, bwd, common + [
        (dict(x=0), INV), (dict(y=0), INV), (dict(dy=0), INV), (dict(dx=0), INV), (dict(dh=0), INV), (dict(g_pre=0), INV), (dict(dg_pre=0), INV),
        (dict(dg_post=0), INV), (dict(g_post=0), INV), (dict(dgate=0), INV), (dict(ws=0), INV), (dict(dxo=0, dh=0, g_pre=0, dg_pre=0), INV),
        (dict(x=P + 1), ALIGN), (dict(dxo=P + 1), ALIGN), (dict(dx=P + 1), ALIGN), (dict(y=P + 2), ALIGN), (dict(dy=P + 2), ALIGN),
        (dict(dh=P + 2), ALIGN), (dict(dgate=P + 2), ALIGN), (dict(ws=P + 64), ALIGN), (dict(n=need - 1), WS)])
    for t, h in ((-1, 8), ((1 << 24) + 1, 8), (4, 0), (4, 16385)):
        assert tq.tq_block_norm_workspace_bytes(t, h) == 0
    assert L.tq_block_norm(*{**good, "t": 0, "x": 0, "y": 0, "x_out": 0, "h_out": 0}.values()) == 0


@host_only
def test_lora_refusals():
    def desc(**k):
        v = dict(n_adapters=3, rank=16, n=100, k=512, type=1, a=P, b=P, scale=None, ranks=None)
        v.update(k)
        return ctypes.byref(tq.tq_adapters(*v.values()))

    bad = [(dict(n_adapters=0), INV), (dict(n_adapters=1025), INV), (dict(rank=0), INV), (dict(rank=12), INV), (dict(rank=136), INV),
           (dict(n=0), INV), (dict(n=(1 << 20) + 1), INV), (dict(k=0), INV), (dict(k=300), INV), (dict(k=16640), INV), (dict(type=3), INV),
           (dict(a=0), INV), (dict(b=0), INV), (dict(a=P + 8), ALIGN), (dict(b=P + 2), ALIGN), (dict(scale=P + 2), ALIGN), (dict(ranks=P + 1), ALIGN)]
    need = int(L.tq_lora_workspace_bytes(desc(), 5))
    assert need > 0
    fwd = dict(ad=desc(), x=P, t=5, ids=P, y=P, out=P, v=P, ws=P, n=need, stream=None)
    refuse(L.tq_lora, fwd, [(dict(ad=desc(**b)), s) for b, s in bad] + [
        (dict(ad=None), INV), (dict(t=-1), INV), (dict(t=(1 << 20) + 1), INV), (dict(x=0), INV), (dict(ids=0), INV), (dict(out=0), INV),
        (dict(ws=0), INV), (dict(x=P + 4), ALIGN), (dict(ids=P + 1), ALIGN), (dict(y=P + 2), ALIGN), (dict(out=P + 2), ALIGN),
        (dict(v=P + 2), ALIGN), (dict(ws=P + 16), ALIGN), (dict(n=need - 1), WS)])
    bwd = dict(ad=desc(), x=P, v=P, dy=P, t=5, ids=P, dx=P, out=P, da=P, db=P, ws=P, n=need, stream=None)
    refuse(L.tq_lora_bwd, bwd, [(dict(ad=desc(**b)), s) for b, s in bad] + [
        (dict(ad=None), INV), (dict(t=-1), INV), (dict(x=0), INV), (dict(v=0), INV), (dict(dy=0), INV), (dict(ids=0), INV), (dict(out=0), INV),
        (dict(da=0), INV), (dict(db=0), INV), (dict(ws=0), INV), (dict(x=P + 8), ALIGN), (dict(dy=P + 2), ALIGN), (dict(da=P + 2), ALIGN),
        (dict(db=P + 2), ALIGN), (dict(dx=P + 1), ALIGN), (dict(out=P + 1), ALIGN), (dict(ws=P + 16), ALIGN), (dict(n=need - 1), WS)])
    # an output over what is still read (the descriptors' pointers are never followed)
    apart = dict(x=P, y=2 * P, out=2 * P, v=3 * P)
    refuse(L.tq_lora, {**fwd, **apart}, [(dict(out=P), INV), (dict(v=P), INV), (dict(v=2 * P), INV)])
    refuse(L.tq_lora_bwd, {**bwd, "v": 2 * P, "dy": 3 * P, "out": 4 * P}, [(dict(out=k * P), INV) for k in (1, 2, 3)])
    for b, s in bad[:11]:
        assert L.tq_lora_workspace_bytes(desc(**b), 5) == 0
    assert L.tq_lora_workspace_bytes(desc(), -1) == 0 and L.tq_lora_workspace_bytes(None, 4) == 0
    assert L.tq_lora(*{**fwd, "t": 0, "x": 0, "out": 0}.values()) == 0


def test_binding_refuses_host_tensors_and_native_half_leaves_them():
    x, i, w = torch.zeros((2, 8)), torch.zeros((2, 2), dtype=torch.int32), torch.zeros((2, 2))
    assert fast.route(x, i, w, None, 0, 0, 0) is None and fast.route(x, i, w) is None
    assert fast.route_balance(x, i, w, None, 0, i, x, x, x, x, 1.0, 0, 0) is None
    assert fast.route_bwd(x, i, w, None, 0, x, None, None, None, 0, 0) is None
    assert fast.weight_grad(x, x, i, w, 3, 0, 0) is None
    assert fast.block_norm(x, x, x, x, None, None, 1.0, None, 1e-6, 0, 0) is None
    assert fast.block_norm(x, None, None, None, None, None, 1, None, 1e-6, 0, 0) is None
    assert fast.block_norm_bwd(x, x, x, x, None, None, 1.0, None, 1e-6, x, x, None, None, None, x, 0, 0) is None
    a = torch.zeros((2, 8, 256))
    assert fast.lora(a, a, None, None, x, i, x, x, None, x, 0, 0) is None
    assert fast.lora_bwd(a, a, None, None, x, i, x, x, a, a, None, None, x, 0, 0) is None
    for f, args in ((tq.tq_route, (x, i, w)), (tq.tq_block_norm, (x, x, x, None)), (tq.tq_moe_weight_grad, (x, x, i, w, 3)),
                    (tq.tq_lora, (tq.TqAdapters(a, a), x, i, x, x))):
        with pytest.raises((TypeError, ValueError)):
            f(*args)


def test_workspaces_grow_with_the_tokens():
    """A workspace of the largest batch holds every smaller one's."""
    ts = sorted({*range(0, 34000, 3), *range(16090, 16110), *(1 << i for i in range(21)), (1 << 20) - 1})
    for na, rank in ((1, 8), (3, 16), (8, 64), (1024, 128)):
        d = ctypes.byref(tq.tq_adapters(na, rank, 100, 512, 1, P, P, None, None))
        need = [int(L.tq_lora_workspace_bytes(d, t)) for t in ts]
        assert need[0] > 0 and need == sorted(need), (na, rank)
    for f, widths in ((tq.tq_route_workspace_bytes, (1, 64, 256, 1000, 4096)), (tq.tq_block_norm_workspace_bytes, (1, 300, 4096, 7168, 16384))):
        for w in widths:
            need = [f(t, w) for t in ts]
            assert need[0] > 0 and need == sorted(need), (f.__name__, w)


@host_only
def test_adapters_refuse_outputs_over_inputs_and_each_other():
    """Any overlap of what a call writes with what it reads or writes elsewhere, but for the in-place forms."""
    t, n, k, r, na = 5, 100, 512, 16, 3
    d = ctypes.byref(tq.tq_adapters(na, r, n, k, 1, P, P, None, None))
    need = int(L.tq_lora_workspace_bytes(d, t))
    at = lambda i: 16 * i * P  # noqa: E731  (far apart)
    end = {"x": at(1) + t * k * 4, "y": at(2) + t * n * 4, "v": at(4) + t * r * 4, "dy": at(2) + t * n * 4}
    fwd = dict(ad=d, x=at(1), t=t, ids=at(6), y=at(2), out=at(3), v=at(4), ws=at(5), n=need, stream=None)
    refuse(L.tq_lora, fwd, [(dict(out=at(1)), INV), (dict(out=end["x"] - 4), INV), (dict(out=at(1) - 4), INV), (dict(out=at(2) + 4), INV),
                            (dict(out=end["y"] - 4), INV), (dict(v=at(2)), INV), (dict(v=at(2) + 8), INV), (dict(v=end["x"] - 4), INV),
                            (dict(v=at(3) + 16), INV), (dict(v=at(2), out=at(2)), INV), (dict(v=end["y"] - 4, out=at(2)), INV)])
    bwd = dict(ad=d, x=at(1), v=at(4), dy=at(2), t=t, ids=at(6), dx=at(7), out=at(8), da=at(9), db=at(10), ws=at(5), n=need, stream=None)
    refuse(L.tq_lora_bwd, bwd, [(dict(out=end["x"] - 4), INV), (dict(out=end["v"] - 4), INV), (dict(out=end["dy"] - 4), INV),
                                (dict(out=at(7) + 4), INV), (dict(da=at(1)), INV), (dict(da=at(4)), INV), (dict(da=at(2)), INV),
                                (dict(da=at(8)), INV), (dict(da=at(7)), INV), (dict(db=at(9)), INV), (dict(db=at(9) + na * r * k * 4 - 4), INV),
                                (dict(db=at(1)), INV), (dict(db=at(4)), INV), (dict(db=at(2)), INV), (dict(db=at(8)), INV)])
