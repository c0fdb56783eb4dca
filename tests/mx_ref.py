"""Plain 64-bit forms of the MXFP4 feed-forward operators (torch on the CPU) and what their tests share."""
from __future__ import annotations

import math

import torch

E2M1 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
SILU, GELU = 0, 1


def quantize(x, noclip=False):
    """(codes 0..15 [t][k], scale bytes [t][k/32]) of a float64 tensor, element by nearest value."""
    t, k = x.shape
    b = x.reshape(-1, 32)
    bad = ~torch.isfinite(b).all(dim=1)
    b = torch.where(bad[:, None], torch.zeros_like(b), b)
    top = b.abs().amax(dim=1)
    m, e = torch.frexp(top)  # top = m 2^e, 0.5 <= m < 1
    e = e.double() - 3 + (m > 0.75) * float(noclip)
    byte = torch.where(top > 0, (e + 127).clamp(0, 254), 0.0)
    r = (b.abs() / 2.0 ** (byte - 127)[:, None]).clamp(max=6.0)
    d = (r[:, :, None] - E2M1).abs()
    near = d == d.amin(dim=2, keepdim=True)
    even = torch.arange(8) % 2 == 0
    c = torch.where((near & even).any(dim=2), (near & even).int().argmax(dim=2), near.int().argmax(dim=2))
    c = c + 8 * torch.signbit(b).long()
    c = torch.where(bad[:, None], 0, c)
    byte = torch.where(bad, 255.0, byte)
    return c.reshape(t, k).to(torch.uint8), byte.reshape(t, k // 32).to(torch.uint8)


def values(c, byte):
    """float64 values of codes [t][k] and scale bytes [t][k/32] (NaN where the byte is 255)."""
    t, k = c.shape
    v = E2M1[(c & 7).long()] * torch.where(c >= 8, -1.0, 1.0)
    s = 2.0 ** (byte.double() - 127)
    s = torch.where(byte == 255, math.nan, s)
    return (v.reshape(t, k // 32, 32) * s[:, :, None]).reshape(t, k)


def pack(c):
    """Codes [t][k] in the layout of the MXFP4 arm: [t][k/256][128]."""
    t, k = c.shape
    b = c.reshape(t, k // 32, 2, 16)
    return (b[:, :, 0] | (b[:, :, 1] << 4)).reshape(t, k // 256, 128).contiguous()


def unpack(codes):
    t, kb, _ = codes.shape
    b = codes.reshape(t, kb * 8, 16)
    return torch.stack([b & 15, b >> 4], dim=2).reshape(t, kb * 256)


def act(kind, z):
    if kind == SILU:
        return z * torch.sigmoid(z)
    # (1 + tanh(b)) / 2 is the logistic function of 2 b, which keeps its small values
    return z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))


def dact(kind, z):
    """act's derivative, written out."""
    if kind == SILU:
        p = torch.sigmoid(z)
        return p + z * p * (1 - p)
    a = math.sqrt(2 / math.pi)
    b = 2 * a * (z + 0.044715 * z ** 3)
    return torch.sigmoid(b) + z * torch.sigmoid(b) * torch.sigmoid(-b) * 2 * a * (1 + 3 * 0.044715 * z * z)


def gated(kind, x, wg, wu, g_add=None, u_add=None):
    g, u = x @ wg.t(), x @ wu.t()
    if g_add is not None:
        g = g + g_add
    if u_add is not None:
        u = u + u_add
    return act(kind, g) * u, g, u


def gated_bwd(kind, g, u, dh):
    return dh * u * dact(kind, g), dh * act(kind, g)


def random_matrix(n, k, gen, spread=4):
    """Random codes and scale bytes around 2^-5, on the CPU."""
    c = torch.randint(0, 16, (n, k), generator=gen, dtype=torch.uint8)
    s = (122 + torch.randint(-spread, spread + 1, (n, k // 32), generator=gen)).to(torch.uint8)
    return c, s
