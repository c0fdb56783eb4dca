"""What the MXFP4 feed-forward operators refuse, before any launch (host only: the device pointers here are made up, so
nothing here may reach a launch)."""
import ctypes

import pytest
import torch

from paper_2608_08910_amd import tq
from test_ops_refusals import ALIGN, INV, L, P, WS, refuse

host_only = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up device pointers; host-only")
G = 1 << 32  # room between made-up tensors


def at(i):
    return P + i * G


def mat(n=64, k=512, codes=at(1), scales=at(2)):
    return ctypes.byref(tq.tq_mat_mx(n, k, codes, scales))


BAD_W = [(dict(n=0), INV), (dict(n=(1 << 20) + 1), INV), (dict(k=0), INV), (dict(k=300), INV), (dict(k=16640), INV), (dict(codes=0), INV),
         (dict(scales=0), INV), (dict(codes=at(1) + 64), ALIGN), (dict(scales=at(2) + 4), ALIGN)]


@host_only
def test_quantize_refusals():
    good = dict(x=at(1), type=1, t=4, k=512, flags=0, codes=at(2), scales=at(3), values=at(4), stream=None)
    refuse(L.tq_quantize_mx, good, [
        (dict(type=3), INV), (dict(type=-1), INV), (dict(t=-1), INV), (dict(t=(1 << 20) + 1), INV), (dict(k=0), INV), (dict(k=100), INV),
        (dict(k=16640), INV), (dict(flags=2), INV), (dict(flags=-1), INV), (dict(x=0), INV), (dict(codes=0), INV), (dict(scales=0), INV),
        (dict(codes=0, scales=0, values=0), INV), (dict(x=at(1) + 8), ALIGN), (dict(codes=at(2) + 64), ALIGN),
        (dict(scales=at(3) + 4), ALIGN), (dict(values=at(4) + 8), ALIGN), (dict(codes=at(1) + 128), INV), (dict(scales=at(1) + 4088), INV),
        (dict(scales=at(2) + 1016), INV), (dict(values=at(1) + 16), INV), (dict(values=at(2) - 4080), INV), (dict(values=at(3)), INV)])
    assert L.tq_quantize_mx(*{**good, "t": 0, "x": 0, "codes": 0, "scales": 0, "values": 0}.values()) == 0


@host_only
def test_gemm_refusals():
    good = dict(w=mat(), x=mat(4, codes=at(3), scales=at(4)), type=0, y=at(5), stream=None)
    refuse(L.tq_gemm_mx, good, [(dict(w=mat(**c)), s) for c, s in BAD_W] + [
        (dict(w=None), INV), (dict(x=None), INV), (dict(x=mat(-1)), INV), (dict(x=mat((1 << 20) + 1)), INV), (dict(x=mat(4, k=256)), INV),
        (dict(x=mat(4, codes=0)), INV), (dict(x=mat(4, scales=0)), INV), (dict(x=mat(4, codes=at(3) + 64)), ALIGN),
        (dict(x=mat(4, scales=at(4) + 2)), ALIGN), (dict(type=3), INV), (dict(y=0), INV), (dict(y=at(5) + 2), ALIGN),
        (dict(y=at(1) + 64 * 256 - 4), INV), (dict(y=at(2) - 1020), INV), (dict(y=at(3)), INV), (dict(y=at(4) + 60), INV)])
    assert L.tq_gemm_mx(*{**good, "x": mat(0, codes=0, scales=0), "y": 0}.values()) == 0


@host_only
def test_gemm_bwd_refusals():
    w = mat()
    need = L.tq_gemm_mx_bwd_workspace_bytes(w, 0, 4)
    assert need > 0
    good = dict(w=w, dy=at(3), type=0, t=4, dx=at(4), ws=at(5), n=need, stream=None)
    refuse(L.tq_gemm_mx_bwd, good, [(dict(w=mat(**c)), s) for c, s in BAD_W] + [
        (dict(w=None), INV), (dict(type=-1), INV), (dict(t=-1), INV), (dict(t=(1 << 20) + 1), INV), (dict(dy=0), INV), (dict(dx=0), INV),
        (dict(ws=0), INV), (dict(dy=at(3) + 2), ALIGN), (dict(dx=at(4) + 1), ALIGN), (dict(ws=at(5) + 128), ALIGN), (dict(n=need - 1), WS),
        (dict(dx=at(3) + 1020), INV), (dict(dx=at(1)), INV), (dict(dx=at(2)), INV), (dict(ws=at(4)), INV), (dict(ws=at(3) - 256), INV),
        (dict(ws=at(1)), INV), (dict(dx=at(5) + need - 4), INV)])
    assert L.tq_gemm_mx_bwd(*{**good, "t": 0, "dy": 0, "dx": 0, "ws": 0}.values()) == 0
    for bad in (mat(n=0), mat(k=100), mat(k=16640), None):
        assert L.tq_gemm_mx_bwd_workspace_bytes(bad, 0, 4) == 0
    for ty, t in ((3, 4), (0, -1), (0, (1 << 20) + 1)):
        assert L.tq_gemm_mx_bwd_workspace_bytes(w, ty, t) == 0


@host_only
def test_gated_refusals():
    up = lambda **c: mat(**{**dict(codes=at(3), scales=at(4)), **c})  # noqa: E731
    x = lambda n=4, **c: mat(n, **{**dict(codes=at(5), scales=at(6)), **c})  # noqa: E731
    good = dict(gate=mat(), up=up(), x=x(), act=0, g_add=at(7), u_add=at(8), type=1, h=at(9), g=at(10), u=at(11), stream=None)
    refuse(L.tq_gated_mx, good, [(dict(gate=mat(**c)), s) for c, s in BAD_W] + [
        (dict(gate=None), INV), (dict(up=None), INV), (dict(x=None), INV), (dict(up=up(n=0)), INV), (dict(up=up(n=65)), INV),
        (dict(up=up(k=256)), INV), (dict(up=up(scales=at(4) + 4)), ALIGN), (dict(x=x(k=256)), INV), (dict(x=x(codes=0)), INV),
        (dict(x=x(-1)), INV), (dict(act=2), INV), (dict(act=-1), INV), (dict(type=3), INV), (dict(h=0), INV), (dict(g=0), INV),
        (dict(u=0), INV), (dict(h=at(9) + 1), ALIGN), (dict(g=at(10) + 1), ALIGN), (dict(u=at(11) + 1), ALIGN),
        (dict(g_add=at(7) + 2), ALIGN), (dict(u_add=at(8) + 2), ALIGN), (dict(g=at(9)), INV), (dict(u=at(9) + 510), INV),
        (dict(u=at(10) - 2), INV), (dict(h=at(7)), INV), (dict(g=at(8) + 1022), INV), (dict(u=at(1)), INV), (dict(h=at(4)), INV),
        (dict(g=at(5)), INV), (dict(h=at(6)), INV)])
    assert L.tq_gated_mx(*{**good, "x": x(0, codes=0, scales=0), "h": 0, "g": 0, "u": 0}.values()) == 0


@host_only
def test_gated_bwd_refusals():
    gate, up = mat(), mat(codes=at(3), scales=at(4))
    need = L.tq_gated_mx_bwd_workspace_bytes(gate, up, 1, 4)
    assert need > 0
    good = dict(gate=gate, up=up, act=0, type=1, t=4, g=at(5), u=at(6), dh=at(7), dg=at(8), du=at(9), dx=at(10), ws=at(11), n=need,
                stream=None)
    refuse(L.tq_gated_mx_bwd, good, [(dict(gate=mat(**c)), s) for c, s in BAD_W] + [
        (dict(gate=None), INV), (dict(up=None), INV), (dict(up=mat(n=65, codes=at(3), scales=at(4))), INV), (dict(act=2), INV),
        (dict(type=3), INV), (dict(t=-1), INV), (dict(t=(1 << 20) + 1), INV), (dict(g=0), INV), (dict(u=0), INV), (dict(dh=0), INV),
        (dict(dg=0), INV), (dict(du=0), INV), (dict(ws=0), INV), (dict(g=at(5) + 1), ALIGN), (dict(u=at(6) + 1), ALIGN),
        (dict(dh=at(7) + 1), ALIGN), (dict(dg=at(8) + 1), ALIGN), (dict(du=at(9) + 1), ALIGN), (dict(dx=at(10) + 1), ALIGN),
        (dict(ws=at(11) + 16), ALIGN), (dict(n=need - 1), WS), (dict(dg=at(9)), INV), (dict(du=at(8) + 2), INV), (dict(dg=at(5) + 2), INV),
        (dict(du=at(7) - 2), INV), (dict(dx=at(5)), INV), (dict(dx=at(7)), INV), (dict(dx=at(8)), INV), (dict(dx=at(9) + 510), INV),
        (dict(dg=at(1)), INV), (dict(du=at(4)), INV), (dict(dx=at(3)), INV), (dict(ws=at(6) - 256), INV), (dict(ws=at(8)), INV),
        (dict(ws=at(10)), INV), (dict(ws=at(2)), INV)])
    assert L.tq_gated_mx_bwd(*{**good, "t": 0, **{n: 0 for n in ("g", "u", "dh", "dg", "du", "dx", "ws")}}.values()) == 0
    for a, b in ((mat(n=0), up), (gate, mat(n=65)), (gate, mat(k=256)), (None, up)):
        assert L.tq_gated_mx_bwd_workspace_bytes(a, b, 1, 4) == 0
    assert L.tq_gated_mx_bwd_workspace_bytes(gate, up, 3, 4) == 0 and L.tq_gated_mx_bwd_workspace_bytes(gate, up, 1, -1) == 0


def test_workspaces_grow_with_the_batch():
    for n, k in ((1, 256), (100, 512), (2048, 4096), (4097, 16384)):
        for ty in (0, 1, 2):
            last = [0, 0]
            for t in (0, 1, 2, 16, 31, 32, 33, 64, 65, 127, 128, 129, 500, 2048, 2049, 8192, 1 << 20):
                now = [L.tq_gemm_mx_bwd_workspace_bytes(mat(n, k), ty, t), L.tq_gated_mx_bwd_workspace_bytes(mat(n, k), mat(n, k), ty, t)]
                assert now[0] >= last[0] and now[1] >= last[1], (n, k, ty, t)
                last = now


@host_only
def test_binding_refuses_host_tensors():
    m = tq.TqMatrixMx(4, 256, torch.zeros(4, 1, 128, dtype=torch.uint8), torch.zeros(4, 8, dtype=torch.uint8))
    x = torch.zeros(4, 256)
    with pytest.raises(TypeError):
        tq.tq_quantize_mx(x, m)
    with pytest.raises(TypeError):
        tq.tq_gemm_mx(m, m, x)
    with pytest.raises(TypeError):
        tq.tq_gemm_mx_bwd(m, x, x, x)
    with pytest.raises(TypeError):
        tq.tq_gated_mx(m, m, m, x)
    with pytest.raises(TypeError):
        tq.tq_gated_mx_bwd(m, m, x, x, x, x, x, x, x)
    with pytest.raises(ValueError):
        tq.tq_quantize_mx(torch.zeros(256), m)
