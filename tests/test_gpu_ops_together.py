"""The router, norms, adapters and the layers' calls together, as a block of a model uses them; on other
streams, captured and replayed, and with workspaces in turns."""
import pytest
import torch

import ops_ref as R
from gpu_util import announce, device

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def tq():
    device()
    from paper_2608_08910_amd import tq as _tq
    return _tq


class Block:
    """norm -> router -> routed experts -> norm, gate, residual, next norm -> projection with adapters,
    and the gradients of the trained parts from given gradients of the stream and of the projection's output."""

    def __init__(self, tq, t, seed=0, hidden=512, inter=256, experts=16, topk=4, n=384, rank=16, na=3):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        rnd = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
        self.tq, self.t, self.topk, self.e = tq, t, topk, experts
        self.ex = tq.TqExperts.empty(experts, hidden, inter)
        for e in range(experts):
            for p in range(3):
                tq.tq_synth_weights(1000 * seed + 3 * e + p, self.ex.matrix(e, p))
        self.proj = tq.TqMatrix.empty(n, hidden)
        tq.tq_synth_weights(77 + seed, self.proj)
        self.ad = tq.TqAdapters((rnd(na, rank, hidden) * hidden ** -0.5).bfloat16(), (rnd(na, n, rank) * 0.1).bfloat16(), rnd(na).abs())
        self.wr = rnd(hidden, experts) * hidden ** -0.5
        self.g1, self.g2, self.g3, self.gate = (1 + 0.1 * rnd(hidden) for _ in range(4))
        self.x = rnd(t, hidden)
        self.ids = torch.randint(-1, na, (t,), device="cuda", dtype=torch.int32, generator=g)
        self.mask = (torch.rand(t, device="cuda", generator=g) < 0.9).to(torch.uint8)
        self.dstream, self.dy = rnd(t, hidden), rnd(t, n)
        new = lambda *s, dtype=F32: torch.zeros(s, device="cuda", dtype=dtype)  # noqa: E731
        self.o = dict(h0=new(t, hidden), idx=new(t, topk, dtype=torch.int32), w=new(t, topk), counts=new(experts, dtype=torch.int32),
                      p_mean=new(experts), coef=new(experts), loss=new(1), y=new(t, hidden), x1=new(t, hidden), h1=new(t, hidden),
                      z=new(t, n), v=new(t, rank), dh1=new(t, hidden), da=new(na, rank, hidden), db=new(na, n, rank), dx=new(t, hidden),
                      dyb=new(t, hidden), dg2=new(hidden), dgate=new(hidden), dg3=new(hidden), dw=new(t, topk), dlogits=new(t, experts))
        self.q, self.d, self.b = new(t, hidden, dtype=torch.int8), new(t, hidden // 256), new(t, hidden // 256, dtype=torch.int32)
        self.one = torch.ones(1, device="cuda")
        self.ws_moe, self.ws_r = tq.moe_workspace(self.ex, t, topk), tq.route_workspace(t, experts)
        self.ws_n, self.ws_l = tq.block_norm_workspace(t, hidden), tq.lora_workspace(self.ad, t)
        self.logits = new(t, experts)

    def forward(self):
        tq, o = self.tq, self.o
        tq.tq_block_norm(self.x, None, None, o["h0"], g_pre=self.g1)
        torch.mm(o["h0"], self.wr, out=self.logits)
        tq.tq_route_balance(self.logits, o["idx"], o["w"], o["counts"], o["p_mean"], o["coef"], o["loss"], self.ws_r, 0.01,
                            token_mask=self.mask, flags=tq.TQ_ROUTE_RENORM)
        tq.tq_moe_grouped(self.ex, o["h0"], o["idx"], o["w"], o["y"], self.ws_moe)
        tq.tq_block_norm(self.x, o["y"], o["x1"], o["h1"], g_post=self.g2, gate=self.gate, res_scale=0.9, g_pre=self.g3)
        tq.tq_gemv_f32(self.proj, o["h1"], o["z"], self.q, self.d, self.b)
        tq.tq_lora(self.ad, o["h1"], self.ids, o["z"], self.ws_l, v=o["v"])

    def backward(self):
        tq, o = self.tq, self.o
        tq.tq_lora_bwd(self.ad, o["h1"], o["v"], self.dy, self.ids, o["da"], o["db"], self.ws_l, out=o["dh1"])
        tq.tq_block_norm_bwd(o["x1"], o["y"], o["dx"], o["dyb"], dx_out=self.dstream, dh=o["dh1"], g_post=self.g2, gate=self.gate,
                             res_scale=0.9, g_pre=self.g3, dg_post=o["dg2"], dgate=o["dgate"], dg_pre=o["dg3"], ws=self.ws_n)
        tq.tq_moe_weight_grad(tq.moe_slot_outputs(self.ex, self.ws_moe, self.t, self.topk), o["dyb"], o["idx"], o["dw"], self.e)
        tq.tq_route_bwd(self.logits, o["idx"], o["w"], o["dlogits"], dw=o["dw"], coef=o["coef"], dloss=self.one, token_mask=self.mask,
                        flags=tq.TQ_ROUTE_RENORM)

    def run(self):
        self.forward()
        self.backward()
        return self.o

    def snapshot(self):
        return {k: v.clone() for k, v in self.o.items()}

    def clear(self):
        for v in self.o.values():
            v.zero_()


@pytest.mark.parametrize("t", [1, 7, 70])
def test_block_against_64_bits(tq, t):
    """Every step from what the step before it left, so that each is held to its own bound; the experts'
    and the projection's own results are taken as they are (they have tests of their own)."""
    announce(f"block t={t}")
    m = Block(tq, t, seed=t)
    m.forward()
    base = m.o["z"].clone()
    tq.tq_gemv_f32(m.proj, m.o["h1"], base, m.q, m.d, m.b)
    m.backward()
    torch.cuda.synchronize()
    c = {k: v.cpu().double() if v.is_floating_point() else v.cpu() for k, v in m.o.items()}
    f = lambda v: v.cpu().double()  # noqa: E731
    u = 64 * R.U
    xo, h, mag = R.block_norm(f(m.x), None, None, None, 1.0, f(m.g1), 1e-6)
    R.close(m.o["h0"], h, u * h.abs() + R.TINY[F32], "h0")
    idx, w, p = R.route(f(m.logits), m.topk, True, m.mask.cpu())
    assert torch.equal(c["idx"].long(), idx)
    R.close(m.o["w"], w, u * w + R.TINY[F32], "w")
    counts, mean, coef, loss = R.balance(idx, p, m.topk, 0.01, m.mask.cpu())
    assert torch.equal(c["counts"].long(), counts)
    R.close(m.o["loss"], loss, u * loss + R.TINY[F32], "loss")
    # a padded token reaches no expert: its stream goes on by itself
    pad = m.mask.cpu() == 0
    assert not bool(m.o["y"].cpu()[pad].any())
    xo, h, mag = R.block_norm(f(m.x), c["y"], f(m.g2), f(m.gate), 0.9, f(m.g3), 1e-6)
    R.close(m.o["x1"], xo, u * mag + R.TINY[F32], "x1")
    R.close(m.o["h1"], h, 4 * u * (h.abs() + R.rfac(xo, 1e-6) * f(m.g3).abs() * mag) + R.TINY[F32], "h1")
    a, b, sc, ids = f(m.ad.a), f(m.ad.b), f(m.ad.scale), m.ids.cpu()
    out, v, omag, vmag = R.lora(a, b, sc, None, c["h1"], ids, f(base))
    R.close(m.o["z"], out, 256 * R.U * omag, "z")
    g = R.lora_bwd(a, b, sc, None, c["h1"], c["v"], f(m.dy), ids, None)
    for k, n in (("da", "da"), ("db", "db"), ("dh1", "out")):
        R.close(m.o[k], g[n][0], (256 + t) * R.U * g[n][1] + R.TINY[F32], k)
    n = R.block_norm_bwd(c["x1"], c["y"], f(m.g2), f(m.gate), 0.9, f(m.g3), 1e-6, f(m.dstream), c["dh1"])
    for k, s in (("dx", "dx"), ("dyb", "dy"), ("dg2", "dg_post"), ("dgate", "dgate"), ("dg3", "dg_pre")):
        R.close(m.o[k], n[s][0], (256 + t) * R.U * n[s][1] + R.TINY[F32], k)
    yd = f(tq.moe_slot_outputs(m.ex, m.ws_moe, t, m.topk)).view(t, m.topk, -1)
    prod = (yd * c["dyb"][:, None]).masked_fill((idx < 0)[..., None], 0.0)
    R.close(m.o["dw"], prod.sum(2), 32 * R.U * prod.abs().sum(2), "dw")
    dl, dmag = R.route_bwd(idx, w, p, True, c["dw"], coef, 1.0)
    R.close(m.o["dlogits"], dl, 4 * u * dmag + R.TINY[F32], "dlogits")


def same(a, b):
    return [k for k in a if not torch.equal(a[k], b[k])]


@pytest.mark.parametrize("t", [1, 33, 600])
def test_another_stream_and_a_replayed_graph(tq, t):
    announce(f"streams and graphs t={t}")
    m = Block(tq, t, seed=50 + t)
    m.run()
    torch.cuda.synchronize()
    want = m.snapshot()
    m.clear()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        m.run()
    s.synchronize()
    assert not same(want, m.o)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        m.run()
    other = Block(tq, t, seed=51 + t)
    other.run()
    torch.cuda.synchronize()
    third = other.snapshot()
    for _ in range(3):  # eager work and synchronizations between the replays
        m.clear()
        graph.replay()
        other.clear()
        other.run()
        torch.cuda.synchronize()
        assert not same(want, m.o) and not same(third, other.o)
    # new inputs under the same graph
    m.x.copy_(other.x * 0.5)
    graph.replay()
    torch.cuda.synchronize()
    replayed = m.snapshot()
    m.clear()
    m.run()
    torch.cuda.synchronize()
    assert not same(replayed, m.o)


def test_two_graphs_share_workspaces_in_order(tq):
    t = 300
    m, k = Block(tq, t, seed=1), Block(tq, t, seed=2)
    for n in ("ws_r", "ws_n", "ws_l"):
        setattr(k, n, getattr(m, n))
    m.run()
    k.run()
    torch.cuda.synchronize()
    want = m.snapshot(), k.snapshot()
    graphs = []
    s = torch.cuda.Stream()
    for z in (m, k):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            z.run()
        graphs.append(g)
    for _ in range(3):
        m.clear()
        k.clear()
        graphs[1].replay()
        graphs[0].replay()
        torch.cuda.synchronize()
        assert not same(want[0], m.o) and not same(want[1], k.o)


def test_explicit_stream_and_bare_pointer(tq):
    """stream= as a stream or its address takes the Python path: the same bits."""
    t, e = 40, 64
    l = torch.randn(t, e, device="cuda")
    a = [torch.zeros(t, 4, dtype=torch.int32, device="cuda"), torch.zeros(t, 4, device="cuda")]
    b = [torch.zeros_like(v) for v in a]
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    tq.tq_route(l, *a, stream=s)
    tq.tq_route(l, *b, stream=s.cuda_stream)
    s.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a, b)) and bool((a[1] > 0).all())


def test_far_offsets(tq):
    """Rows past 2^31 elements from the start (int64 addressing): the last rows of a long batch."""
    t, h = (1 << 31) // 16384 + 40, 16384
    if torch.cuda.get_device_properties(0).total_memory < 100 << 30:
        pytest.skip("needs 40 GB")
    x = torch.empty((t, h), dtype=torch.bfloat16, device="cuda")
    x[-50:] = torch.randn(50, h, device="cuda").bfloat16()
    x[:-50] = 1.0
    g = torch.ones(h, device="cuda")
    out = torch.empty_like(x)
    tq.tq_block_norm(x, None, None, out, g_pre=g)
    want = torch.empty((50, h), dtype=torch.bfloat16, device="cuda")
    tq.tq_block_norm(x[-50:].clone(), None, None, want, g_pre=g)
    torch.cuda.synchronize()
    assert torch.equal(out[-50:], want)
    del x, out
    e = 2048
    t = (1 << 31) // e + 40
    l = torch.zeros((t, e), dtype=torch.bfloat16, device="cuda")
    l[-50:] = torch.randn(50, e, device="cuda").bfloat16()
    idx, w = torch.empty((t, 4), dtype=torch.int32, device="cuda"), torch.empty((t, 4), device="cuda")
    tq.tq_route(l, idx, w)
    i2, w2 = torch.empty((50, 4), dtype=torch.int32, device="cuda"), torch.empty((50, 4), device="cuda")
    tq.tq_route(l[-50:].clone(), i2, w2)
    torch.cuda.synchronize()
    assert torch.equal(idx[-50:], i2) and torch.equal(w[-50:], w2)


def test_more_threads_than_a_launch_takes(tq):
    """The most tokens: 2^24 rows past 256 columns, and 2^26 slots, are more than 2^32 threads (the last rows and those around
    2^23, of a stream that is otherwise ones, against those of short calls)."""
    if torch.cuda.get_device_properties(0).total_memory < 200 << 30:
        pytest.skip("needs 100 GB")
    t, h = 1 << 24, 513
    announce(f"block_norm t={t} h={h}")
    x = torch.ones((t, h), dtype=torch.bfloat16, device="cuda")
    g = 1 + 0.1 * torch.randn(h, device="cuda")
    gate = torch.rand(t, 1, device="cuda")
    out, nxt = torch.empty_like(x), torch.empty_like(x)
    spots = [(0, 8), ((1 << 23) - 8, (1 << 23) + 8), (t - 8, t)]  # (rows a multiple of four apart have their sums' order in common)
    for a, b in spots:
        x[a:b] = torch.randn(b - a, h, device="cuda").bfloat16()
    tq.tq_block_norm(x, x, out, nxt, g_post=g, gate=gate, g_pre=g)
    for a, b in spots:
        o, n = torch.empty_like(out[a:b]), torch.empty_like(out[a:b])
        tq.tq_block_norm(x[a:b].clone(), x[a:b].clone(), o, n, g_post=g, gate=gate[a:b].clone(), g_pre=g)
        torch.cuda.synchronize()
        assert torch.equal(o, out[a:b]) and torch.equal(n, nxt[a:b])
    del x, out, nxt
    t, topk, h = 1 << 20, 64, 256
    announce(f"weight_grad t={t} topk={topk} h={h}")
    yd = torch.empty((t * topk, h), device="cuda")
    dout = torch.randn(t, h, device="cuda")
    yd.fill_(1.0)
    idx = torch.zeros((t, topk), dtype=torch.int32, device="cuda")
    dw = torch.full((t, topk), -77.0, device="cuda")
    spots = [(0, 40), (t // 2 - 40, t // 2 + 40), (t - 40, t)]
    for a, b in spots:
        yd[a * topk:b * topk] = torch.randn((b - a) * topk, h, device="cuda")
    tq.tq_moe_weight_grad(yd, dout, idx, dw, 4)
    for a, b in spots:
        s = torch.empty(b - a, topk, device="cuda")
        tq.tq_moe_weight_grad(yd[a * topk:b * topk].clone(), dout[a:b].clone(), idx[a:b].clone(), s, 4)
        torch.cuda.synchronize()
        assert torch.equal(s, dw[a:b])
    assert not bool((dw == -77.0).any())


@pytest.mark.parametrize("t", [1, 7, 70, 600])
def test_weight_gradient_of_the_layers_output(tq, t):
    """The layer's output is linear in its routing weights: with the weight 1 on one slot of each token it is that slot's part, and
    the gradient is its product with the output's gradient (formed from the call with the block's own weights)."""
    announce(f"weight gradient of the layer t={t}")
    m = Block(tq, t, seed=90 + t)
    m.forward()
    o = m.o
    dout = torch.randn(t, o["y"].shape[1], device="cuda")
    tq.tq_moe_weight_grad(tq.moe_slot_outputs(m.ex, m.ws_moe, t, m.topk), dout, o["idx"], o["dw"], m.e)
    dw = o["dw"].clone()
    for j in range(m.topk):
        one = torch.zeros_like(o["w"])
        one[:, j] = 1.0
        y = torch.empty_like(o["y"])
        tq.tq_moe_grouped(m.ex, o["h0"], o["idx"], one, y, m.ws_moe)
        torch.cuda.synchronize()
        prod = y.cpu().double() * dout.cpu().double()
        # (a lane adds hidden / 64 products one after the other, then 8 additions join the lanes)
        R.close(dw[:, j], prod.sum(1), (prod.shape[1] / 64 + 10) * R.U * prod.abs().sum(1), f"dw {j}")
