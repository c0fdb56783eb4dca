"""Norms around a block and their gradients on the GPU against the plain 64-bit forms."""
import pytest
import torch

import ops_ref as R
from gpu_util import announce, device

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
RS, EPS = 0.75, 1e-5


@pytest.fixture(scope="module")
def tq():
    device()
    from paper_2608_08910_amd import tq as _tq
    return _tq


def make(t, h, xt, yt, gate, post, pre, block, seed):
    g = torch.Generator().manual_seed(seed + 31 * t + h)
    rnd = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    v = {"x": (3 * rnd(t, h) * torch.where(torch.rand(h, generator=g) < 0.05, 10.0, 1.0)).to(xt),
         "y": (rnd(t, h) * torch.exp(2 * rnd(t, 1))).to(yt) if block else None,
         "g_post": 1 + 0.3 * rnd(h) if block and post else None, "g_pre": 1 + 0.3 * rnd(h) if pre else None,
         "gate": {None: None, "channel": rnd(h), "token": rnd(t, 1)}[gate] if block else None,
         "dxo": rnd(t, h).to(xt), "dh": rnd(t, h).to(yt) if pre else None}
    if block and t > 1:
        v["y"][t // 2] = 0  # a token for which no expert answered
    return v


def dev(v, off):
    return {k: None if z is None else R.offset(z, off if k in ("x", "y", "dxo", "dh") else 0) for k, z in v.items()}


SHAPES = [(1, 1), (2, 3), (3, 64), (5, 255), (1, 256), (4, 257), (7, 1000), (3, 1024), (2, 1027), (6, 2048), (3, 2049), (5, 4096),
          (2, 4099), (1, 7168), (3, 7168), (2, 8191), (2, 8193), (3, 16383), (2, 16384), (1100, 64), (600, 520), (520, 5000)]
FORMS = [("channel", True, True, True), ("token", True, True, True), (None, False, True, True), ("channel", False, False, True),
         ("token", True, False, True), (None, True, True, False)]
TYPES = [(F32, F32), (BF16, F32), (BF16, BF16), (F16, F32), (F16, F16)]


def bounds(v, h):
    """Half steps per value. A mean square adds at most 16 squares in a thread, 8 steps in the wave
    and up to 16 waves, all positive, and enters through a root (half of it); the factors of a term
    are a handful more."""
    return 40 * R.U


@pytest.mark.parametrize("n,shape", list(enumerate(SHAPES)))
def test_block_norm(tq, n, shape):
    t, h = shape
    for f, (gate, post, pre, block) in enumerate(FORMS):
        xt, yt = TYPES[(n + f) % 5]
        announce(f"block_norm t={t} h={h} {xt} {yt} gate={gate} post={post} pre={pre} block={block}")
        v = make(t, h, xt, yt, gate, post, pre, block, 1)
        d = dev(v, (n + f) % 3)
        z = {k: None if a is None else a.double() for k, a in v.items()}
        xo, hh, mag = R.block_norm(z["x"], z["y"], z["g_post"], z["gate"], RS, z["g_pre"], EPS)
        g = R.Guards()
        x_out = g.new((t, h), xt, off=n % 2) if block else None
        ho = g.new((t, h), yt, off=f % 2) if pre else None
        tq.tq_block_norm(d["x"], d["y"], x_out, ho, g_post=d["g_post"], gate=d["gate"], res_scale=RS, g_pre=d["g_pre"], eps=EPS)
        torch.cuda.synchronize()
        g.check()
        b = bounds(v, h)
        if block:
            R.close(x_out, xo, b * mag + R.HALF[xt] * xo.abs() * (1 + b) + R.TINY[xt], "x_out")
        if pre:
            # x_out's own error, and what it moves the mean square by
            spread = mag.norm(dim=1, keepdim=True) / xo.norm(dim=1, keepdim=True).clamp(min=1e-300)
            fac = R.rfac(xo, EPS) * z["g_pre"].abs()
            R.close(ho, hh, b * fac * mag + b * (2 + spread) * hh.abs() + R.HALF[yt] * hh.abs() + R.TINY[yt], "h")


@pytest.mark.parametrize("n,shape", list(enumerate(SHAPES)))
def test_block_norm_bwd(tq, n, shape):
    t, h = shape
    for f, (gate, post, pre, block) in enumerate(FORMS):
        for have in ("both", "stream", "next"):
            if (have == "next" and not pre) or (have == "stream" and (pre or not block)):
                continue
            xt, yt = TYPES[(n + f) % 5]
            announce(f"block_norm_bwd t={t} h={h} {xt} {yt} gate={gate} post={post} pre={pre} block={block} {have}")
            v = make(t, h, xt, yt, gate, post, pre, block, 2)
            if have == "next":
                v["dxo"] = None
            d = dev(v, (n + f) % 3)
            z = {k: None if a is None else a.double() for k, a in v.items()}
            ref = R.block_norm_bwd(z["x"], z["y"], z["g_post"], z["gate"], RS, z["g_pre"], EPS, z["dxo"], z["dh"])
            g = R.Guards()
            o = {"dx": g.new((t, h), xt, off=n % 2), "dy": g.new((t, h), yt, off=f % 2) if block else None}
            for k, src in (("dg_post", "g_post"), ("dgate", "gate"), ("dg_pre", "g_pre")):
                o[k] = None if v[src] is None else g.new(tuple(v[src].shape))
            ws = tq.block_norm_workspace(t, h)
            tq.tq_block_norm_bwd(d["x"] if pre else None, d["y"], o["dx"], o["dy"], dx_out=d["dxo"], dh=d["dh"], g_post=d["g_post"],
                                 gate=d["gate"], res_scale=RS, g_pre=d["g_pre"], eps=EPS, dg_post=o["dg_post"], dgate=o["dgate"],
                                 dg_pre=o["dg_pre"], ws=ws)
            torch.cuda.synchronize()
            g.check()
            assert set(ref) == {k for k in o if o[k] is not None}
            for k, (want, mag) in ref.items():
                # two means in a row, each 40 half steps and its factors; a sum over tokens adds them
                # one by one in a workgroup and its workgroups in rows of 16
                adds = 0 if k in ("dx", "dy") else t / 256 + 48
                ty = {"dx": xt, "dy": yt}.get(k, F32)
                R.close(o[k], want, (160 + adds) * R.U * mag + R.HALF[ty] * want.abs() + R.TINY[ty], k)


def test_in_place_and_equal_bits(tq):
    v = make(37, 4096, F32, F32, "channel", True, True, True, 3)
    d = dev(v, 0)
    kw = dict(g_post=d["g_post"], gate=d["gate"], res_scale=RS, g_pre=d["g_pre"], eps=EPS)
    x_out, h = torch.empty_like(d["x"]), torch.empty_like(d["y"])
    tq.tq_block_norm(d["x"], d["y"], x_out, h, **kw)
    res = []
    for _ in range(2):
        o = {k: torch.empty_like(d[s]) for k, s in (("dx", "x"), ("dy", "y"), ("dg_post", "g_post"), ("dgate", "gate"), ("dg_pre", "g_pre"))}
        tq.tq_block_norm_bwd(x_out, d["y"], o["dx"], o["dy"], dx_out=d["dxo"], dh=d["dh"], dg_post=o["dg_post"], dgate=o["dgate"],
                             dg_pre=o["dg_pre"], ws=tq.block_norm_workspace(37, 4096), **kw)
        res.append(o)
    assert all(torch.equal(res[0][k], res[1][k]) for k in res[0])
    dxo, dh = d["dxo"].clone(), d["dh"].clone()
    tq.tq_block_norm_bwd(x_out, d["y"], dxo, dh, dx_out=dxo, dh=dh, dg_post=o["dg_post"], dgate=o["dgate"], dg_pre=o["dg_pre"],
                         ws=tq.block_norm_workspace(37, 4096), **kw)
    assert torch.equal(dxo, res[0]["dx"]) and torch.equal(dh, res[0]["dy"])
    x, y = d["x"].clone(), d["y"].clone()
    tq.tq_block_norm(x, y, x, y, **kw)
    assert torch.equal(x, x_out) and torch.equal(y, h)


# several rows a workgroup and rows that begin at every place of a four; the widest ones; rows shorter than a four
ODD = [(300, 4093), (1030, 255), (270, 4097), (261, 8190), (259, 12001), (258, 16381), (257, 16382), (700, 2), (1025, 5), (9, 4094)]


@pytest.mark.parametrize("n,shape", list(enumerate(ODD)))
def test_odd_rows(tq, n, shape):
    test_block_norm(tq, n, shape)
    test_block_norm_bwd(tq, n, shape)


@pytest.mark.parametrize("t,h", [(530, 1001), (300, 12001), (2, 3)])
def test_odd_rows_in_place(tq, t, h):
    v = make(t, h, BF16, BF16, "channel", True, True, True, 4)
    d = dev(v, 0)
    kw = dict(g_post=d["g_post"], gate=d["gate"], res_scale=RS, g_pre=d["g_pre"], eps=EPS)
    x_out, hh = torch.empty_like(d["x"]), torch.empty_like(d["y"])
    tq.tq_block_norm(d["x"], d["y"], x_out, hh, **kw)
    x, y = d["x"].clone(), d["y"].clone()
    tq.tq_block_norm(x, y, x, y, **kw)
    assert torch.equal(x, x_out) and torch.equal(y, hh)
    gr = {k: torch.empty_like(d[s]) for k, s in (("dg_post", "g_post"), ("dgate", "gate"), ("dg_pre", "g_pre"))}
    dx, dy, ws = torch.empty_like(x), torch.empty_like(y), tq.block_norm_workspace(t, h)
    tq.tq_block_norm_bwd(x_out, d["y"], dx, dy, dx_out=d["dxo"], dh=d["dh"], ws=ws, **gr, **kw)
    dxo, dh = d["dxo"].clone(), d["dh"].clone()
    tq.tq_block_norm_bwd(x_out, d["y"], dxo, dh, dx_out=dxo, dh=dh, ws=ws, **gr, **kw)
    assert torch.equal(dxo, dx) and torch.equal(dh, dy)


def test_no_tokens(tq):
    z = lambda *s: torch.empty(s, device="cuda")  # noqa: E731
    g = R.Guards()
    gp, ga, gr = g.new((100,)), g.new((100,)), g.new((100,))
    w = torch.ones(100, device="cuda")
    tq.tq_block_norm(z(0, 100), z(0, 100), z(0, 100), z(0, 100), g_post=w, gate=w, g_pre=w)
    tq.tq_block_norm_bwd(z(0, 100), z(0, 100), z(0, 100), z(0, 100), dx_out=z(0, 100), dh=z(0, 100), g_post=w, gate=w, g_pre=w,
                         dg_post=gp, dgate=ga, dg_pre=gr, ws=tq.block_norm_workspace(0, 100))
    torch.cuda.synchronize()
    g.check()
    assert not bool(gp.any() or ga.any() or gr.any())


# rows of every magnitude whose squares fp32 holds, with rows of zeros: the rsqrt factors go from 1e-16 to 1e15
MAGNITUDES = [1e16, 1.0, 1e-14, 0.0, 1e15, 1e14, 0.0, 1e-10, 1e12]


@pytest.mark.parametrize("eps", [1e-30, 1e-6, 1.0])
@pytest.mark.parametrize("t,h", [(18, 64), (9, 520), (300, 1001), (9, 4099), (9, 7168), (9, 12004)])
def test_far_magnitudes(tq, t, h, eps):
    for f, (gate, post, pre, block) in enumerate(FORMS):
        for have in ("both", "stream", "next"):
            if (have == "next" and not pre) or (have == "stream" and (pre or not block)):
                continue
            xt, yt = ((F32, F32), (BF16, F32), (BF16, BF16))[f % 3]
            announce(f"far magnitudes t={t} h={h} eps={eps} {xt} {yt} gate={gate} post={post} pre={pre} block={block} {have}")
            v = make(t, h, xt, yt, gate, post, pre, block, 6)
            s = torch.tensor([MAGNITUDES[i % 9] for i in range(t)])[:, None]
            v["x"] = (v["x"].float() * s).to(xt)
            if block:  # (the magnitudes in another order; both are zero in row 3)
                v["y"] = (v["y"].float() * torch.tensor([MAGNITUDES[(2 * i + 6) % 9] for i in range(t)])[:, None]).to(yt)
                v["y"][3::9] = 0
                # (three rows of the drawn 300 pass the documented range: their squares sum to 4.6e38, 1.6e39 and 1.7e39)
                v["y"][(v["y"].double() ** 2).sum(1) > 3.4e38] *= 2.0 ** -10
            if have == "next":
                v["dxo"] = None
            d = dev(v, f % 3)
            z = {k: None if a is None else a.double() for k, a in v.items()}
            ref = R.block_norm_bwd(z["x"], z["y"], z["g_post"], z["gate"], RS, z["g_pre"], eps, z["dxo"], z["dh"])
            g = R.Guards()
            o = {"dx": g.new((t, h), xt), "dy": g.new((t, h), yt) if block else None}
            for k, src in (("dg_post", "g_post"), ("dgate", "gate"), ("dg_pre", "g_pre")):
                o[k] = None if v[src] is None else g.new(tuple(v[src].shape))
            tq.tq_block_norm_bwd(d["x"] if pre else None, d["y"], o["dx"], o["dy"], dx_out=d["dxo"], dh=d["dh"], g_post=d["g_post"],
                                 gate=d["gate"], res_scale=RS, g_pre=d["g_pre"], eps=eps, dg_post=o["dg_post"], dgate=o["dgate"],
                                 dg_pre=o["dg_pre"], ws=tq.block_norm_workspace(t, h))
            torch.cuda.synchronize()
            g.check()
            for k, (want, mag) in ref.items():  # (the bound of test_block_norm_bwd)
                adds = 0 if k in ("dx", "dy") else t / 256 + 48
                ty = {"dx": xt, "dy": yt}.get(k, F32)
                R.close(o[k], want, (160 + adds) * R.U * mag + R.HALF[ty] * want.abs() + R.TINY[ty], k)


@pytest.mark.parametrize("h", [64, 1001, 7168, 12004])
def test_an_infinite_block_output_without_a_norm_after_it(tq, h):
    """Without g_post, dy = gate * D: what y holds does not enter."""
    announce(f"infinite y h={h}")
    t = 6
    v = make(t, h, F32, F32, "channel", False, False, True, 7)
    v["y"][2, 5], v["y"][4, h - 1] = float("inf"), float("nan")
    d = dev(v, 0)
    g = R.Guards()
    dx, dy, dgate = g.new((t, h)), g.new((t, h)), g.new((h,))
    tq.tq_block_norm_bwd(None, d["y"], dx, dy, dx_out=d["dxo"], gate=d["gate"], res_scale=RS, dgate=dgate, eps=EPS,
                         ws=tq.block_norm_workspace(t, h))
    torch.cuda.synchronize()
    g.check()
    # (one product each)
    assert torch.equal(dx, d["dxo"] * RS) and torch.equal(dy, d["dxo"] * d["gate"])
