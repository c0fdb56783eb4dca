"""The native half of the binding of the router, block norms and adapters takes exactly the calls that the
Python path takes, with the same results and the same refusals."""
import pytest
import torch

from paper_2608_08910_amd import _tqpy as fast
from paper_2608_08910_amd import tq
from test_native_binding import outcome

pytestmark = pytest.mark.gpu
CALLS = ["route", "route_balance", "route_bwd", "weight_grad", "block_norm", "block_norm_bwd", "lora", "lora_bwd"]


def args_of(name):
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    r = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    t, e, k, h = 6, 20, 3, 256
    idx = torch.argsort(torch.rand(t, e, device="cuda", generator=g), dim=1)[:, :k].to(torch.int32).contiguous()
    mask = torch.ones(t, dtype=torch.uint8, device="cuda")
    if name == "route":
        return lambda a, b, c, m: tq.tq_route(a, b, c, m, 1), [r(t, e).bfloat16(), idx, r(t, k), mask]
    if name == "route_balance":
        f = lambda a, b, c, m, n, p, q, s, ws: (tq.tq_route_balance(a, b, c, n, p, q, s, ws, 0.5, m), ws.zero_())  # noqa: E731
        return f, [r(t, e), idx, r(t, k), mask, torch.zeros(e, dtype=torch.int32, device="cuda"), r(e), r(e), r(1),
                   torch.zeros_like(tq.route_workspace(t, e))]
    if name == "route_bwd":
        f = lambda a, b, c, m, dl, dw, co, ds: tq.tq_route_bwd(a, b, c, dl, dw, co, ds, m)  # noqa: E731
        return f, [r(t, e).half(), idx, torch.rand(t, k, device="cuda", generator=g), mask, torch.zeros(t, e, device="cuda").half(), r(t, k), r(e), r(1)]
    if name == "weight_grad":
        return lambda *a: tq.tq_moe_weight_grad(*a, 20), [r(t * k, h), r(t, h), idx, r(t, k)]
    x, y = r(t, h).bfloat16(), r(t, h)
    if name == "block_norm":
        f = lambda x, y, o, n, gp, ga, gr: tq.tq_block_norm(x, y, o, n, gp, ga, 0.5, gr)  # noqa: E731
        return f, [x, y, torch.zeros_like(x), torch.zeros_like(y), r(h), r(h), r(h)]
    if name == "block_norm_bwd":
        def f(x, y, dx, dy, do, dh, gp, ga, gr, dgp, dga, dgr, ws):
            tq.tq_block_norm_bwd(x, y, dx, dy, do, dh, gp, ga, 0.5, gr, 1e-6, dgp, dga, dgr, ws)
            ws.zero_()
        return f, [x, y, torch.zeros_like(x), torch.zeros_like(y), r(t, h).bfloat16(), r(t, h), r(h), r(t, 1), r(h), r(h), r(t, 1), r(h),
                   torch.zeros_like(tq.block_norm_workspace(t, h))]
    n, rank = 70, 8
    a, b, sc, rk = r(2, rank, h), r(2, n, rank), r(2), torch.tensor([8, 5], dtype=torch.int32, device="cuda")
    ids = torch.tensor([0, 1, -1, 1, 0, 2], dtype=torch.int32, device="cuda")
    ws = torch.zeros_like(tq.lora_workspace(tq.TqAdapters(a, b), t))
    if name == "lora":
        f = lambda a, b, sc, rk, x, i, y, o, v, ws: (tq.tq_lora(tq.TqAdapters(a, b, sc, rk), x, i, y, ws, o, v), ws.zero_())  # noqa: E731
        return f, [a, b, sc, rk, r(t, h), ids, r(t, n), r(t, n), r(t, rank), ws]
    f = lambda a, b, sc, rk, x, i, v, dy, da, db, dx, o, ws: (  # noqa: E731
        tq.tq_lora_bwd(tq.TqAdapters(a, b, sc, rk), x, v, dy, i, da, db, ws, dx, o), ws.zero_())
    return f, [a, b, sc, rk, r(t, h), ids, r(t, rank), r(t, n), torch.zeros_like(a), torch.zeros_like(b), r(t, h), r(t, h), ws]


@pytest.mark.parametrize("name", CALLS)
def test_native_and_python_paths_agree(name, monkeypatch):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.init()
    _, args = args_of(name)
    variants = [lambda a: a]
    for i in range(len(args)):
        variants += [lambda a, i=i: a[:i] + [a[i].double()] + a[i + 1:],
                     lambda a, i=i: a[:i] + [a[i].narrow(-1, 0, 1)] + a[i + 1:],
                     lambda a, i=i: a[:i] + [a[i].transpose(0, -1)] + a[i + 1:],
                     lambda a, i=i: a[:i] + [a[i].cpu()] + a[i + 1:],
                     lambda a, i=i: a[:i] + [a[i][None]] + a[i + 1:],
                     lambda a, i=i: a[:i] + [None] + a[i + 1:]]
    taken = 0
    for j, v in enumerate(variants):
        res = []
        for native in (True, False):
            monkeypatch.setattr(tq, "_fast", fast if native else None)
            fn, args = args_of(name)
            res.append(outcome(fn, v(list(args))))
        if isinstance(res[0], list):
            taken += 1
            assert all(torch.equal(p, r) for p, r in zip(*res)), f"{name} variant {j}"
        else:
            assert res[0] == res[1], f"{name} variant {j}"
    assert taken > 0
    calls = []
    real = getattr(fast, name)

    class Spy:
        def __getattr__(self, a):
            def f(*x):
                calls.append(real(*x))
                return calls[-1]
            return f
    monkeypatch.setattr(tq, "_fast", Spy())
    fn, args = args_of(name)
    fn(*args)
    assert calls == [0], "a plain call takes the native path"
