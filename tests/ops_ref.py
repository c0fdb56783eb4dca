"""Plain 64-bit forms of the router, the block norms and the low-rank adapters (torch on the CPU, loops
where they say it most plainly), with their gradients written out, and what the GPU tests share."""
from __future__ import annotations

import math

import torch

U = 2.0 ** -24  # half a step of fp32, relative
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
# half the distance between a type's smallest values (below them a rounding is absolute)
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}


# ---- guards: tensors inside a larger buffer whose rest must stay as it was --------------------

class Guards:
    def __init__(self, device="cuda"):
        self.bufs, self.device = [], device

    def new(self, shape, dtype=torch.float32, off=0):
        """An uninitialised tensor of this shape, `off` elements past a 256-byte boundary."""
        n = math.prod(shape)
        pad = 256
        b = torch.full((pad + n + off + pad,), 77, dtype=dtype, device=self.device)
        self.bufs.append((b, pad + off, n))
        return b[pad + off:pad + off + n].view(shape)

    def check(self):
        for b, at, n in self.bufs:
            assert bool((b[:at] == 77).all()) and bool((b[at + n:] == 77).all()), "written outside a tensor"


def offset(t: torch.Tensor, off: int) -> torch.Tensor:
    """A contiguous device copy of t that starts `off` elements past an aligned address."""
    b = torch.empty(t.numel() + off + 8, dtype=t.dtype, device="cuda")
    v = b[off:off + t.numel()].view(t.shape)
    v.copy_(t)
    return v


def close(got, ref, bound, what):
    got, ref, bound = got.detach().cpu().double(), ref.double(), bound.double().expand(ref.shape)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    same = (got == ref) | (torch.isnan(got) & torch.isnan(ref))
    bad = ~((got - ref).abs() <= bound) & ~same
    if bool(bad.any()):
        i = int(torch.where(bad, (got - ref).abs() / bound.clamp(min=1e-300), 0.0).nan_to_num(nan=1e300).argmax())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off; at {i}: got {got.flatten()[i]!r}, "
                             f"ref {ref.flatten()[i]!r}, bound {bound.flatten()[i]!r}")


# ---- router --------------------------------------------------------------------------------------

def route(logits, topk, renorm, mask=None):
    """(idx [t][k] int64, w, p) of float64 logits, token by token."""
    t, e = logits.shape
    idx, w, p = torch.full((t, topk), -1), torch.zeros((t, topk), dtype=torch.float64), torch.zeros((t, e), dtype=torch.float64)
    for i in range(t):
        row = logits[i]
        if (mask is not None and not mask[i]) or bool((row == -math.inf).all()):
            continue
        ex = torch.exp(row - row.max())
        p[i] = ex / ex.sum()
        order = sorted((x for x in range(e) if row[x] > -math.inf), key=lambda x: (-float(row[x]), x))[:topk]
        idx[i, :len(order)] = torch.tensor(order)
        w[i, :len(order)] = ex[order] / (ex[order].sum() if renorm else ex.sum())
    return idx, w, p


def balance(idx, p, topk, alpha, mask=None):
    """(counts, p_mean, coef, loss)."""
    e = p.shape[1]
    tv = p.shape[0] if mask is None else int((mask != 0).sum())
    counts = torch.bincount(idx[idx >= 0], minlength=e)
    if tv == 0:
        z = torch.zeros(e, dtype=torch.float64)
        return counts, z, z, torch.zeros(1, dtype=torch.float64)
    mean, f = p.sum(0) / tv, counts.double()
    return counts, mean, alpha * e * f / (topk * tv * tv), (alpha * e / (topk * tv) * (f * mean).sum()).reshape(1)


def route_bwd(idx, w, p, renorm, dw, coef, dloss):
    """dlogits and the sum of its absolute terms."""
    t, e = p.shape
    out, mag = torch.zeros_like(p), torch.zeros_like(p)
    for i in range(t):
        if coef is not None:
            c = dloss * coef
            out[i] += p[i] * (c - (p[i] * c).sum())
            mag[i] += p[i] * (c.abs() + (p[i] * c.abs()).sum())
        if dw is None:
            continue
        on = idx[i] >= 0
        s, sa = (w[i] * dw[i])[on].sum(), (w[i] * dw[i]).abs()[on].sum()
        for j in range(idx.shape[1]):
            if on[j]:
                x = idx[i, j]
                f = w[i, j] if renorm else p[i, x]
                out[i, x] += f * (dw[i, j] - s) if renorm else f * dw[i, j]
                mag[i, x] += f * (dw[i, j].abs() + sa)
        if not renorm:
            out[i] -= p[i] * s
            mag[i] += p[i] * sa
    return out, mag


# ---- block norms -----------------------------------------------------------------------------------

def rfac(v, eps):
    return 1.0 / torch.sqrt((v * v).mean(1, keepdim=True) + eps)


def block_norm(x, y, g_post, gate, rs, g_pre, eps):
    """(x_out, h or None, sum of absolute terms of x_out)."""
    if y is None:
        xo, mag = x, x.abs()
    else:
        n = y * rfac(y, eps) * g_post if g_post is not None else y
        n = n * gate if gate is not None else n
        xo, mag = rs * x + n, (rs * x).abs() + n.abs()
    return xo, (None if g_pre is None else xo * rfac(xo, eps) * g_pre), mag


def block_norm_bwd(xo, y, g_post, gate, rs, g_pre, eps, dxo, dh):
    """{name: (gradient, sum of absolute terms)}."""
    o = {}
    some = dxo if dxo is not None else dh
    D, M = (torch.zeros_like(some), torch.zeros_like(some)) if dxo is None else (dxo, dxo.abs())
    if dh is not None:
        r = rfac(xo, eps)
        q = dh * g_pre
        D = D + r * (q - xo * r * r * (q * xo).mean(1, keepdim=True))
        M = M + r * (q.abs() + xo.abs() * r * r * (q * xo).abs().mean(1, keepdim=True))
        o["dg_pre"] = ((dh * xo * r).sum(0), (dh * xo * r).abs().sum(0))
    if y is None:
        o["dx"] = (D, M)
        return o
    o["dx"] = (rs * D, abs(rs) * M)
    ga = gate if gate is not None else torch.ones(1, dtype=torch.float64)
    dn, dm = ga * D, ga.abs() * M
    if g_post is not None:
        r = rfac(y, eps)
        q, qm = dn * g_post, dm * g_post.abs()
        o["dy"] = (r * (q - y * r * r * (q * y).mean(1, keepdim=True)),
                   r * (qm + y.abs() * r * r * (qm * y.abs()).mean(1, keepdim=True)))
        o["dg_post"] = ((dn * y * r).sum(0), (dm * (y * r).abs()).sum(0))
        n = y * r * g_post
    else:
        o["dy"], n = (dn, dm), y
    if gate is not None:
        ax = 0 if gate.dim() == 1 else 1
        o["dgate"] = ((D * n).sum(ax, keepdim=ax == 1), (M * n.abs()).sum(ax, keepdim=ax == 1))
    return o


# ---- low-rank adapters -------------------------------------------------------------------------------

def _each(ids, a, ranks):
    na, R, _ = a.shape
    for i in range(ids.numel()):
        g = int(ids[i])
        if 0 <= g < na:
            r = R if ranks is None else max(0, min(R, int(ranks[g])))
            yield i, g, r


def lora(a, b, scale, ranks, x, ids, y):
    """(out, v, magnitude of out, magnitude of v)."""
    R, n = a.shape[1], b.shape[1]
    out = torch.zeros((ids.numel(), n), dtype=torch.float64) if y is None else y.clone()
    mag = out.abs()
    v, vm = (torch.zeros((ids.numel(), R), dtype=torch.float64) for _ in range(2))
    for i, g, r in _each(ids, a, ranks):
        s = 1.0 if scale is None else scale[g]
        v[i, :r], vm[i, :r] = a[g, :r] @ x[i], a[g, :r].abs() @ x[i].abs()
        out[i] += s * (b[g, :, :r] @ v[i, :r])
        mag[i] += abs(s) * (b[g, :, :r].abs() @ vm[i, :r])
    return out, v, mag, vm


def lora_bwd(a, b, scale, ranks, x, v, dy, ids, dx):
    """{name: (gradient, magnitude)} with da, db, out."""
    da, dam, db, dbm = (torch.zeros_like(z) for z in (a, a, b, b))
    out = torch.zeros_like(x) if dx is None else dx.clone()
    mag = out.abs()
    for i, g, r in _each(ids, a, ranks):
        s = 1.0 if scale is None else scale[g]
        u, um = s * (b[g, :, :r].t() @ dy[i]), abs(s) * (b[g, :, :r].abs().t() @ dy[i].abs())
        da[g, :r] += torch.outer(u, x[i])
        dam[g, :r] += torch.outer(um, x[i].abs())
        db[g, :, :r] += s * torch.outer(dy[i], v[i, :r])
        dbm[g, :, :r] += abs(s) * torch.outer(dy[i].abs(), v[i, :r].abs())
        out[i] += a[g, :r].t() @ u
        mag[i] += a[g, :r].abs().t() @ um
    return {"da": (da, dam), "db": (db, dbm), "out": (out, mag)}
