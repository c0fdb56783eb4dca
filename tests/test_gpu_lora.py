"""Low-rank adapters of many requests and their gradients on the GPU against the plain 64-bit forms."""
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


def make(t, n, k, rank, na, dtype, pick, seed=0, scale=True, ranks=True):
    g = torch.Generator().manual_seed(seed + t + n + k + rank)
    rnd = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    v = {"a": (rnd(na, rank, k) * k ** -0.5).to(dtype), "b": (rnd(na, n, rank) * 0.1).to(dtype),
         "scale": rnd(na) if scale else None, "ranks": None, "x": rnd(t, k), "y": rnd(t, n), "dy": rnd(t, n), "dx": rnd(t, k)}
    if ranks:
        v["ranks"] = torch.randint(0, rank + 1, (na,), generator=g, dtype=torch.int32)
        v["ranks"][0] = rank + 5  # (clamped)
        if na > 1:
            v["ranks"][1] = -2
        for i in range(na):  # storage past the live ranks may hold anything
            r = max(0, min(rank, int(v["ranks"][i])))
            v["a"][i, r:] = math.nan
            v["b"][i, :, r:] = math.inf
    ids = torch.randint(-1, na + 1, (t,), generator=g, dtype=torch.int32)
    if pick == "one":
        ids[:] = na - 1
    elif pick == "none":
        ids[:] = -1
    elif pick == "runs":
        ids = ids.sort().values
    elif pick == "skew":
        ids = torch.where(torch.rand(t, generator=g) < 0.8, 0, ids).to(torch.int32)
    v["ids"] = ids
    v["x"][(ids < 0) | (ids >= na)] = math.nan  # not read
    return v


def clean(v):
    """64-bit copies, with what is not read zeroed."""
    z = {k: a.double().nan_to_num(nan=0.0, posinf=0.0) if a is not None and a.is_floating_point() else a for k, a in v.items()}
    return z


CASES = [  # t, n, k, rank, adapters, type, pick
    (1, 1, 256, 8, 1, F32, "one"), (1, 4096, 4096, 16, 8, BF16, "one"), (1, 100, 16384, 64, 2, F16, "one"),
    (2, 257, 512, 24, 3, BF16, "any"), (3, 64, 256, 128, 5, F32, "any"), (32, 2048, 1024, 16, 64, BF16, "any"),
    (64, 333, 768, 40, 7, F16, "skew"), (65, 333, 768, 40, 7, F16, "skew"), (66, 1, 256, 8, 1, BF16, "one"),
    (70, 65, 512, 16, 100, F32, "any"), (100, 1000, 256, 32, 3, BF16, "none"), (129, 4097, 512, 64, 4, BF16, "runs"),
    (200, 192, 1280, 104, 6, F16, "any"), (300, 130, 256, 128, 2, F32, "skew"), (517, 70, 2048, 16, 9, BF16, "any"),
    (1030, 48, 256, 8, 1024, BF16, "any"), (1100, 300, 256, 48, 1, F32, "one"),
    # one launch over several columns a thread, and its tokens without an adapter; tiles of every type and rank step
    (2, 5000, 1024, 8, 2, F32, "any"), (30, 1025, 256, 16, 4, F16, "none"), (1200, 40, 512, 8, 5, F16, "runs"),
    (1300, 257, 2304, 16, 3, F32, "skew"), (1090, 70, 1024, 24, 40, BF16, "any"), (1150, 515, 256, 72, 3, F16, "runs"),
    (1500, 64, 768, 128, 2, BF16, "skew"), (1027, 36, 8192, 64, 30, BF16, "any"), (1040, 2, 256, 112, 2, F32, "any")]


@pytest.mark.parametrize("t,n,k,rank,na,dtype,pick", CASES)
def test_lora_and_gradient(tq, t, n, k, rank, na, dtype, pick):
    announce(f"lora t={t} n={n} k={k} rank={rank} adapters={na} {dtype} {pick}")
    v = make(t, n, k, rank, na, dtype, pick, scale=t % 2 == 0, ranks=pick != "one" or t > 1000)
    z = clean(v)
    d = {s: None if a is None else R.offset(a, 1 if s in ("y", "dy", "ids") else 0) for s, a in v.items()}
    ad = tq.TqAdapters(d["a"], d["b"], d["scale"], d["ranks"])
    ref, low, mag, lmag = R.lora(z["a"], z["b"], z["scale"], z["ranks"], z["x"], z["ids"], z["y"])
    g = R.Guards()
    out, vv, ws = g.new((t, n), off=1), g.new((t, rank)), tq.lora_workspace(ad, t)
    tq.tq_lora(ad, d["x"], d["ids"], d["y"], ws, out=out, v=vv)
    torch.cuda.synchronize()
    g.check()
    # a chain of additions over k is at most k / 8 long (eight waves share it; few tokens: k / 64), joins add at
    # most 16, and the second product's chain is the rank
    kb = k / 8 + 20
    R.close(vv, low, kb * R.U * lmag + R.TINY[F32], "v")
    R.close(out, ref, (kb + rank + 8) * R.U * mag, "out")
    none = (z["ids"] < 0) | (z["ids"] >= na)
    assert torch.equal(out.cpu()[none], v["y"][none])
    # in place, with nothing else kept
    y2 = d["y"].clone()
    tq.tq_lora(ad, d["x"], d["ids"], y2, ws)
    assert torch.equal(y2, out)
    # by itself
    alone = g.new((t, n))
    tq.tq_lora(ad, d["x"], d["ids"], None, ws, out=alone)
    R.close(alone, ref - z["y"], (kb + rank + 8) * R.U * mag, "out alone")

    gref = R.lora_bwd(z["a"], z["b"], z["scale"], z["ranks"], z["x"], low, z["dy"], z["ids"], z["dx"])
    o = {"da": g.new((na, rank, k)), "db": g.new((na, n, rank), off=1), "out": g.new((t, k), off=1)}
    low32 = low.float().cuda()
    tq.tq_lora_bwd(ad, d["x"], low32, d["dy"], d["ids"], o["da"], o["db"], ws, dx=d["dx"], out=o["out"])
    torch.cuda.synchronize()
    g.check()
    # u: a chain over n as above; the sums over tokens: at most a token per addition
    nb = n / 8 + 24
    R.close(o["da"], gref["da"][0], (nb + t + 16) * R.U * gref["da"][1] + R.TINY[F32], "da")
    R.close(o["db"], gref["db"][0], (t + 20) * R.U * gref["db"][1] + R.TINY[F32], "db")
    R.close(o["out"], gref["out"][0], (nb + rank + 8) * R.U * gref["out"][1], "dx")
    dx2, da2, db2 = d["dx"].clone(), torch.empty_like(o["da"]), torch.empty_like(o["db"])
    tq.tq_lora_bwd(ad, d["x"], low32, d["dy"], d["ids"], da2, db2, ws, dx=dx2)
    assert torch.equal(dx2, o["out"]) and torch.equal(da2, o["da"]) and torch.equal(db2, o["db"])
    da2.fill_(7)
    tq.tq_lora_bwd(ad, d["x"], low32, d["dy"], d["ids"], da2, db2, ws)
    assert torch.equal(da2, o["da"])


def test_no_tokens(tq):
    v = make(1, 40, 256, 8, 3, BF16, "one")
    ad = tq.TqAdapters(v["a"].cuda(), v["b"].cuda())
    e = lambda *s, dtype=F32: torch.empty(s, dtype=dtype, device="cuda")  # noqa: E731
    g = R.Guards()
    da, db = g.new((3, 8, 256)), g.new((3, 40, 8))
    ws = tq.lora_workspace(ad, 0)
    tq.tq_lora(ad, e(0, 256), e(0, dtype=torch.int32), e(0, 40), ws)
    tq.tq_lora_bwd(ad, e(0, 256), e(0, 8), e(0, 40), e(0, dtype=torch.int32), da, db, ws)
    torch.cuda.synchronize()
    g.check()
    assert not bool(da.any()) and not bool(db.any())


@pytest.mark.parametrize("na,rank", [(3, 16), (8, 64)])
def test_a_workspace_of_a_longer_batch(tq, na, rank):
    """One workspace, of the largest batch, serves every smaller one, with the bits of a workspace of its own."""
    big, n, k = 16384, 36, 512
    v = make(big, n, k, rank, na, BF16, "any", seed=7, ranks=False)
    d = {s: None if a is None else a.cuda() for s, a in v.items()}
    ad = tq.TqAdapters(d["a"], d["b"], d["scale"])
    ws = tq.lora_workspace(ad, big)
    for t in (1, 5, 100, 200, 1100, 8100, 16000, big):
        announce(f"lora, workspace of {big} tokens for {t}, adapters={na} rank={rank}")
        got = []
        for w in (ws, tq.lora_workspace(ad, t)):
            o = [torch.empty(t, n, device="cuda"), torch.empty(t, rank, device="cuda"), torch.empty(na, rank, k, device="cuda"),
                 torch.empty(na, n, rank, device="cuda"), torch.empty(t, k, device="cuda")]
            tq.tq_lora(ad, d["x"][:t], d["ids"][:t], d["y"][:t], w, out=o[0], v=o[1])
            tq.tq_lora_bwd(ad, d["x"][:t], o[1], d["dy"][:t], d["ids"][:t], o[2], o[3], w, out=o[4])
            torch.cuda.synchronize()
            got.append(o)
        none = (d["ids"][:t] < 0) | (d["ids"][:t] >= na)
        assert all(torch.equal(a, b) for a, b in zip(*got)) and torch.equal(got[0][0][none], d["y"][:t][none])


def by_adapter(v, z, low=None):
    """The forms of ops_ref an adapter's tokens at a time, with the sums of absolute terms: (out, v, their magnitudes), and with
    `low` (the forward call's v) the gradients as well."""
    na, rank, k = z["a"].shape
    out, mag = z["y"].clone(), z["y"].abs()
    lo, lm = (torch.zeros((z["ids"].numel(), rank), dtype=torch.float64) for _ in range(2))
    gr = {"da": torch.zeros_like(z["a"]), "db": torch.zeros_like(z["b"]), "out": z["dx"].clone()}
    gm = {"da": torch.zeros_like(z["a"]), "db": torch.zeros_like(z["b"]), "out": z["dx"].abs()}
    for g in range(na):
        tok = torch.nonzero(z["ids"] == g).flatten()
        r = rank if z["ranks"] is None else max(0, min(rank, int(z["ranks"][g])))
        s = 1.0 if z["scale"] is None else float(z["scale"][g])
        if not tok.numel() or not r:
            continue
        a, b, x, dy = z["a"][g, :r], z["b"][g, :, :r].contiguous(), z["x"][tok], z["dy"][tok]
        at, bt = a.t().contiguous(), b.t().contiguous()
        lo[tok, :r], lm[tok, :r] = x @ at, x.abs() @ at.abs()
        out[tok] += s * (lo[tok, :r] @ bt)
        mag[tok] += abs(s) * (lm[tok, :r] @ bt.abs())
        if low is not None:
            u, um = s * (dy @ b), abs(s) * (dy.abs() @ b.abs())
            gr["da"][g, :r], gm["da"][g, :r] = u.t().contiguous() @ x, um.t().contiguous() @ x.abs()
            w = low[tok, :r]
            gr["db"][g, :, :r], gm["db"][g, :, :r] = s * (dy.t().contiguous() @ w), abs(s) * (dy.abs().t().contiguous() @ w.abs())
            gr["out"][tok] += u @ a
            gm["out"][tok] += um @ a.abs()
    return (out, lo, mag, lm) if low is None else (gr, gm)


# several turns of columns a workgroup in the second product (rows of fours and odd ones); ids past what the plan keeps in
# registers; first products in 4, 3, 2 and 1 parts
LONG = [(2100, 8192, 256, 64, 3, BF16, "any"), (2100, 8191, 512, 24, 2, F32, "skew"), (4200, 4097, 256, 40, 5, F16, "runs"),
        (5000, 40, 1024, 8, 70, BF16, "any"), (9000, 36, 1536, 8, 4, F32, "runs"), (9900, 1027, 256, 16, 3, F16, "any"),
        (12000, 33, 2048, 16, 6, BF16, "skew"), (33000, 20, 512, 8, 2, BF16, "any")]


@pytest.mark.parametrize("t,n,k,rank,na,dtype,pick", LONG)
def test_many_tokens(tq, t, n, k, rank, na, dtype, pick):
    announce(f"lora, many tokens t={t} n={n} k={k} rank={rank} adapters={na} {dtype} {pick}")
    v = make(t, n, k, rank, na, dtype, pick, seed=3)
    z = clean(v)
    ref, low, mag, lmag = by_adapter(v, z)
    d = {s: None if a is None else a.cuda() for s, a in v.items()}
    ad = tq.TqAdapters(d["a"], d["b"], d["scale"], d["ranks"])
    g = R.Guards()
    out, vv, ws = g.new((t, n), off=1), g.new((t, rank)), tq.lora_workspace(ad, t)
    tq.tq_lora(ad, d["x"], d["ids"], d["y"], ws, out=out, v=vv)
    torch.cuda.synchronize()
    g.check()
    # a chain of additions is at most the whole sum, and a few joins
    R.close(vv, low, (k + 20) * R.U * lmag + R.TINY[F32], "v")
    R.close(out, ref, (k + rank + 28) * R.U * mag, "out")
    none = (z["ids"] < 0) | (z["ids"] >= na)
    assert torch.equal(out.cpu()[none], v["y"][none])
    gref, gmag = by_adapter(v, z, low)
    o = {"da": g.new((na, rank, k)), "db": g.new((na, n, rank)), "out": g.new((t, k))}
    tq.tq_lora_bwd(ad, d["x"], low.float().cuda(), d["dy"], d["ids"], o["da"], o["db"], ws, dx=d["dx"], out=o["out"])
    torch.cuda.synchronize()
    g.check()
    R.close(o["da"], gref["da"], (n + t + 40) * R.U * gmag["da"] + R.TINY[F32], "da")
    R.close(o["db"], gref["db"], (t + 20) * R.U * gmag["db"] + R.TINY[F32], "db")
    R.close(o["out"], gref["out"], (n + rank + 32) * R.U * gmag["out"], "dx")


@pytest.mark.parametrize("t,n,k,rank,na,dtype", [(9, 1100, 512, 16, 3, BF16), (50, 300, 768, 40, 3, F32), (1200, 300, 768, 40, 3, BF16),
                                                 (1100, 65, 512, 16, 2, F16), (1300, 64, 256, 128, 4, F32)])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_bad_token_stays_by_itself(tq, t, n, k, rank, na, dtype, bad):
    """A NaN or infinity in x or dy of a token with an adapter: in its own row, and in its adapter's gradients, alone."""
    announce(f"lora, bad token t={t} n={n} k={k} rank={rank} adapters={na} {dtype} {bad}")
    v = make(t, n, k, rank, na, dtype, "any", seed=5, ranks=False)
    tok = t - 2
    v["ids"][tok] = 1
    v["ids"][tok - 1], v["ids"][tok + 1] = 1, 0
    d = {s: None if a is None else a.cuda() for s, a in v.items()}
    d["x"].nan_to_num_(nan=1.0)
    ad = tq.TqAdapters(d["a"], d["b"], d["scale"])
    ws = tq.lora_workspace(ad, t)

    def run():
        o = {"out": torch.zeros(t, n, device="cuda"), "v": torch.zeros(t, rank, device="cuda"), "da": torch.zeros(na, rank, k, device="cuda"),
             "db": torch.zeros(na, n, rank, device="cuda"), "dx": torch.zeros(t, k, device="cuda")}
        tq.tq_lora(ad, d["x"], d["ids"], d["y"], ws, out=o["out"], v=o["v"])
        tq.tq_lora_bwd(ad, d["x"], o["v"], d["dy"], d["ids"], o["da"], o["db"], ws, dx=d["dx"], out=o["dx"])
        torch.cuda.synchronize()
        return o

    want = run()
    keep = torch.arange(t, device="cuda") != tok
    others = torch.arange(na, device="cuda") != 1
    x0 = d["x"].clone()
    d["x"][tok, k // 2 + 3] = bad
    got = run()
    for s in ("out", "v"):
        assert torch.equal(got[s][keep], want[s][keep]) and not bool(torch.isfinite(got[s][tok]).any()), s
    for s in ("da", "db"):
        assert torch.equal(got[s][others], want[s][others]) and not bool(torch.isfinite(got[s][1]).all()), s
    assert torch.equal(got["dx"], want["dx"])
    d["x"].copy_(x0)
    d["dy"][tok, n // 2] = bad
    got = run()
    assert torch.equal(got["out"], want["out"]) and torch.equal(got["v"], want["v"])
    assert torch.equal(got["dx"][keep], want["dx"][keep]) and not bool(torch.isfinite(got["dx"][tok]).any())
    for s in ("da", "db"):
        assert torch.equal(got[s][others], want[s][others]) and not bool(torch.isfinite(got[s][1]).all()), s


def test_far_offsets(tq):
    """Rows past 2^31 elements from the start, in either matrix's width: the last rows against those of a short call."""
    if torch.cuda.get_device_properties(0).total_memory < 100 << 30:
        pytest.skip("needs 60 GB")
    for t, n, k in (((1 << 31) // 16384 + 40, 8, 16384), (2090, 1 << 20, 256)):
        announce(f"lora, far offsets t={t} n={n} k={k}")
        g = torch.Generator(device="cuda").manual_seed(t)
        rnd = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
        ad = tq.TqAdapters((rnd(1, 8, k) * k ** -0.5).bfloat16(), (rnd(1, n, 8) * n ** -0.5).bfloat16())
        x, dy = torch.ones(t, k, device="cuda"), torch.ones(t, n, device="cuda")
        x[-40:], dy[-40:] = rnd(40, k), rnd(40, n)
        ids = torch.zeros(t, dtype=torch.int32, device="cuda")
        out, v, dx = torch.empty(t, n, device="cuda"), torch.empty(t, 8, device="cuda"), torch.empty(t, k, device="cuda")
        da, db, ws = torch.empty(1, 8, k, device="cuda"), torch.empty(1, n, 8, device="cuda"), tq.lora_workspace(ad, t)
        tq.tq_lora(ad, x, ids, None, ws, out=out, v=v)
        tq.tq_lora_bwd(ad, x, v, dy, ids, da, db, ws, out=dx)
        torch.cuda.synchronize()
        a, b = ad.a[0].double(), ad.b[0].double()
        xl, dyl = x[-40:].double(), dy[-40:].double()
        low, u = xl @ a.t().contiguous(), dyl @ b
        lm, um = xl.abs() @ a.t().contiguous().abs(), dyl.abs() @ b.abs()
        bt = b.t().contiguous()
        R.close(v[-40:], low.cpu(), (k + 20) * R.U * lm.cpu(), "v")
        R.close(out[-40:], (low @ bt).cpu(), (k + 40) * R.U * (lm @ bt.abs()).cpu(), "out")
        R.close(dx[-40:], (u @ a).cpu(), (n + 40) * R.U * (um @ a.abs()).cpu(), "dx")
        del x, dy, out, dx
