"""Timed cases of the MXFP4 feed-forward block: quantisation to MXFP4, products of MXFP4 rows with
frozen MXFP4 weights, the gated block in one pass, and the gradients of both by their inputs.

Kinds:
  quantize   `tq_quantize_mx`: rows -> e2m1 codes, e8m0 scales and the values that they stand for.
  gemm       `tq_gemm_mx`: y[t][n] = X W^T, both operands in MXFP4.
  gemm_bwd   `tq_gemm_mx_bwd`: dx[t][k] = dy W, W in MXFP4.
  gated      `tq_gated_mx`: h = act(X Wg^T + g_add) * (X Wu^T + u_add), where `save` with the two
             pre-activations that the backward pass reads.
  gated_bwd  `tq_gated_mx_bwd`: dg, du (rounded to the type) and dx = dg Wg + du Wu.

MXFP4 rows are uint8 tensors: codes [rows][k/256][128], where byte i of a 16-byte piece holds element i of a
block of 32 in its low and element 16 + i in its high nibble, and scales [rows][k/32].

With `own` false, `run` computes the same outputs from elementary torch operations in fp32.
"""
import math

import torch

own = False


# ------------------------------------------------------------------------------------
# the cases
# ------------------------------------------------------------------------------------

def listed():
    return [
        # the smallest call: one decoded token's activations
        {"name": "quantize_h4096_t1", "kind": "quantize", "k": 4096, "t": 1, "type": "bf16", "noclip": False},
        # a ragged training batch of the deep model's width, with the values for the straight-through pass
        {"name": "quantize_h7168_t4091", "kind": "quantize", "k": 7168, "t": 4091, "type": "bf16", "noclip": False},
        # one decoded token's down projection
        {"name": "gemm_4096x2048_t1", "kind": "gemm", "n": 4096, "k": 2048, "t": 1, "type": "f32"},
        # a decode batch on a decode step's stacked rows
        {"name": "gemm_32768x4096_t32", "kind": "gemm", "n": 32768, "k": 4096, "t": 32, "type": "bf16"},
        # a ragged prefill chunk's down projection on the deep model's width
        {"name": "gemm_7168x2048_t2043", "kind": "gemm", "n": 7168, "k": 2048, "t": 2043, "type": "bf16"},
        # the gradient of a small batch's projection in the framework's own activation type
        {"name": "gemm_bwd_2048x4096_t33", "kind": "gemm_bwd", "n": 2048, "k": 4096, "t": 33, "type": "f32"},
        # the gradient of a training batch's down projection
        {"name": "gemm_bwd_4096x2048_t2048", "kind": "gemm_bwd", "n": 4096, "k": 2048, "t": 2048, "type": "bf16"},
        # one decoded token through a shared expert of the deep model
        {"name": "gated_h7168_i2048_t1", "kind": "gated", "n": 2048, "k": 7168, "t": 1, "type": "bf16", "act": "silu",
         "save": False, "add": False},
        # a decode batch through a shared expert
        {"name": "gated_h4096_i2048_t32", "kind": "gated", "n": 2048, "k": 4096, "t": 32, "type": "bf16", "act": "silu",
         "save": False, "add": False},
        # a training batch through a dense layer: adapters' parts added, pre-activations kept
        {"name": "gated_h7168_i16384_t4096", "kind": "gated", "n": 16384, "k": 7168, "t": 4096, "type": "bf16",
         "act": "silu", "save": True, "add": True},
        # the gradients of a ragged training batch through a shared expert, and of a long one
        {"name": "gated_bwd_h4096_i2048_t2047", "kind": "gated_bwd", "n": 2048, "k": 4096, "t": 2047, "type": "bf16",
         "act": "silu"},
        {"name": "gated_bwd_h7168_i2048_t8192", "kind": "gated_bwd", "n": 2048, "k": 7168, "t": 8192, "type": "bf16",
         "act": "gelu"},
    ]


def _logint(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


_TYPES = ["f32", "bf16", "bf16", "f16"]


def draw(rng):
    kind = rng.choice(["quantize"] * 2 + ["gemm"] * 3 + ["gemm_bwd"] * 3 + ["gated"] * 4 + ["gated_bwd"] * 3)
    if kind == "quantize":
        k = 256 * _logint(rng, 1, 64)
        return {"kind": kind, "k": k, "t": _logint(rng, 1, max(1, 4091 * 7168 // k)), "type": rng.choice(_TYPES),
                "noclip": rng.random() < 0.3}
    while True:
        c = {"kind": kind, "n": _logint(rng, 64, 32768), "k": 256 * _logint(rng, 1, 64), "t": _logint(rng, 1, 8192),
             "type": rng.choice(_TYPES)}
        if kind in ("gated", "gated_bwd"):
            c["n"] = (c["n"] + 1) // 2
            c["act"] = rng.choice(["silu", "gelu"])
        if kind == "gated":
            c["save"], c["add"] = rng.random() < 0.5, rng.random() < 0.3
        if c["t"] * c["n"] * c["k"] <= 4096 * 4096 * 4096 and c["n"] * c["k"] <= 16384 * 8192:
            return c


# ------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------

_DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(9000011 * int(seed) + 29)
    return g


def _randn(g, *shape):
    return torch.randn(shape, device="cuda", generator=g)


def _rand(g, *shape):
    return torch.rand(shape, device="cuda", generator=g)


def _acts(g, t, k):
    """Activations after a norm: a few large channels, tokens of different magnitude, some rows of padding."""
    big = torch.where(_rand(g, k) < 0.01, 20.0, 1.0)
    x = _randn(g, t, k) * big * torch.exp(0.7 * (2 * _rand(g, t, 1) - 1))
    return torch.where(_rand(g, t, 1) < 0.02, 0.0, x) if t > 1 else x


def _weights(g, n, k):
    return _quantized(_randn(g, n, k) * (k ** -0.5) * torch.exp(0.5 * _randn(g, n, 1)))


def _draw_quantize(c, g):
    return {"x": _acts(g, c["t"], c["k"]).to(_DT[c["type"]])}


def _draw_gemm(c, g):
    return {"w": _weights(g, c["n"], c["k"]), "xq": _quantized(_acts(g, c["t"], c["k"]))}


def _draw_gemm_bwd(c, g):
    return {"w": _weights(g, c["n"], c["k"]), "dy": (_randn(g, c["t"], c["n"]) * 0.02).to(_DT[c["type"]])}


def _draw_gated(c, g):
    t, n, k = c["t"], c["n"], c["k"]
    s = {"gate": _weights(g, n, k), "up": _weights(g, n, k), "xq": _quantized(_acts(g, t, k)), "g_add": None,
         "u_add": None}
    if c["add"]:
        s["g_add"], s["u_add"] = _randn(g, t, n) * 0.1, _randn(g, t, n) * 0.1
    return s


def _draw_gated_bwd(c, g):
    t, n, k = c["t"], c["n"], c["k"]
    dt = _DT[c["type"]]
    # pre-activations as a block has them: the gate's mostly small, some far out on both sides
    return {"gate": _weights(g, n, k), "up": _weights(g, n, k), "g": (_randn(g, t, n) * 2).to(dt),
            "u": _randn(g, t, n).to(dt), "dh": (_randn(g, t, n) * 0.02).to(dt)}


_DRAW = {"quantize": _draw_quantize, "gemm": _draw_gemm, "gemm_bwd": _draw_gemm_bwd, "gated": _draw_gated,
         "gated_bwd": _draw_gated_bwd}


def prepare(case, seed):
    s = _DRAW[case["kind"]](case, _gen(seed))
    s["case"] = case
    if own:
        from paper_2608_08910_amd import tq
        _buffers(tq, case, s)
    return s


def _buffers(tq, c, s):
    """Matrix handles, outputs and workspaces that a program keeps from call to call."""
    kind, t, k, dt = c["kind"], c["t"], c["k"], _DT[c["type"]]

    def new(*shape):
        return torch.empty(shape, dtype=dt, device="cuda")
    for name in ("w", "gate", "up", "xq"):
        if name in s:
            codes, scales = s[name]
            s["m_" + name] = tq.TqMatrixMx(codes.shape[0], k, codes, scales)
    if kind == "quantize":
        s["m"], s["values"] = tq.TqMatrixMx.empty(t, k), new(t, k)
        s["flags"] = tq.TQ_MX_NOCLIP if c["noclip"] else 0
    elif kind == "gemm":
        s["y"] = new(t, c["n"])
    elif kind == "gemm_bwd":
        s["dx"], s["ws"] = new(t, k), tq.gemm_mx_bwd_workspace(s["m_w"], t, dt)
    else:
        s["act"] = {"silu": tq.TQ_ACT_SILU, "gelu": tq.TQ_ACT_GELU}[c["act"]]
        if kind == "gated":
            s["h"] = new(t, c["n"])
            s["g"], s["u"] = (new(t, c["n"]), new(t, c["n"])) if c["save"] else (None, None)
        else:
            s["dg"], s["du"], s["dx"] = new(t, c["n"]), new(t, c["n"]), new(t, k)
            s["ws"] = tq.gated_mx_bwd_workspace(s["m_gate"], s["m_up"], t, dt)


# ------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------

def run(state):
    kind = state["case"]["kind"]
    if own:
        return _OWN[kind](state)
    return _PLAIN[kind](state)


def _own_quantize(s):
    from paper_2608_08910_amd import tq
    tq.tq_quantize_mx(s["x"], s["m"], values=s["values"], flags=s["flags"])
    return {"codes": s["m"].codes, "scales": s["m"].scales, "values": s["values"]}


def _own_gemm(s):
    from paper_2608_08910_amd import tq
    tq.tq_gemm_mx(s["m_w"], s["m_xq"], s["y"])
    return {"y": s["y"]}


def _own_gemm_bwd(s):
    from paper_2608_08910_amd import tq
    tq.tq_gemm_mx_bwd(s["m_w"], s["dy"], s["dx"], s["ws"])
    return {"dx": s["dx"]}


def _own_gated(s):
    from paper_2608_08910_amd import tq
    tq.tq_gated_mx(s["m_gate"], s["m_up"], s["m_xq"], s["h"], act=s["act"], g_add=s["g_add"], u_add=s["u_add"], g=s["g"],
                   u=s["u"])
    return {k: s[k] for k in ("h", "g", "u") if s[k] is not None}


def _own_gated_bwd(s):
    from paper_2608_08910_amd import tq
    tq.tq_gated_mx_bwd(s["m_gate"], s["m_up"], s["g"], s["u"], s["dh"], s["dg"], s["du"], s["dx"], s["ws"], act=s["act"])
    return {k: s[k] for k in ("dg", "du", "dx")}


_OWN = {"quantize": _own_quantize, "gemm": _own_gemm, "gemm_bwd": _own_gemm_bwd, "gated": _own_gated,
        "gated_bwd": _own_gated_bwd}

_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _scale_bytes(b, noclip):
    """e8m0 bytes of blocks b [..., 32]: the largest magnitude's exponent less 2, one more where `noclip` and
    6 times that scale does not reach it."""
    top = b.abs().amax(dim=-1)
    m, e = torch.frexp(top)  # top = m 2^e, 0.5 <= m < 1
    e = e + 124
    if noclip:
        e = e + (m > 0.75).to(e.dtype)
    return torch.where(top > 0, e.clamp(0, 254), 0)


def _quantized(x, noclip=False):
    """(codes, scales) of rows x [t][k]; finite and within 2^-100 .. 2^100 of zero."""
    t, k = x.shape
    b = x.float().reshape(t, k // 32, 32)
    e = _scale_bytes(b, noclip)
    r = b.abs() * torch.exp2((127 - e).clamp(max=127).float())[..., None]
    c = ((r > 0.25).to(torch.uint8) + (r >= 0.75) + (r > 1.25) + (r >= 1.75) + (r > 2.5) + (r >= 3.5) + (r > 5.0))
    c = c + 8 * torch.signbit(b).to(torch.uint8)
    codes = c[..., :16] + 16 * c[..., 16:]
    return codes.to(torch.uint8).reshape(t, k // 256, 128), e.to(torch.uint8)


def _values(q):
    """fp32 values [rows][k] of (codes, scales)."""
    codes, scales = q
    rows, nb = scales.shape
    p = codes.reshape(rows, nb, 16).int()
    table = torch.tensor(_E2M1 + [-v for v in _E2M1], device="cuda")
    v = torch.cat([table[p & 15], table[p >> 4]], dim=2)
    return (v * torch.exp2(scales.float() - 127.0)[..., None]).reshape(rows, nb * 32)


def _p_quantize(s):
    q = _quantized(s["x"], s["case"]["noclip"])
    return {"codes": q[0], "scales": q[1], "values": _values(q).to(s["x"].dtype)}


def _p_gemm(s):
    return {"y": (_values(s["xq"]) @ _values(s["w"]).t()).to(_DT[s["case"]["type"]])}


def _p_gemm_bwd(s):
    return {"dx": (s["dy"].float() @ _values(s["w"])).to(s["dy"].dtype)}


_GELU_A, _GELU_B = math.sqrt(2 / math.pi), 0.044715


def _p_gated(s):
    c = s["case"]
    x = _values(s["xq"])
    g, u = x @ _values(s["gate"]).t(), x @ _values(s["up"]).t()
    if c["add"]:
        g, u = g + s["g_add"], u + s["u_add"]
    if c["act"] == "silu":
        a = g / (1 + torch.exp(-g))
    else:
        a = 0.5 * g * (1 + torch.tanh(_GELU_A * (g + _GELU_B * g * g * g)))
    dt = _DT[c["type"]]
    o = {"h": (a * u).to(dt)}
    if c["save"]:
        o["g"], o["u"] = g.to(dt), u.to(dt)
    return o


def _p_gated_bwd(s):
    c = s["case"]
    g, u, dh = s["g"].float(), s["u"].float(), s["dh"].float()
    if c["act"] == "silu":
        p = 1 / (1 + torch.exp(-g))
        a, da = g * p, p * (1 + g * (1 - p))
    else:
        th = torch.tanh(_GELU_A * (g + _GELU_B * g * g * g))
        a = 0.5 * g * (1 + th)
        da = 0.5 * (1 + th) + 0.5 * g * (1 - th) * (1 + th) * _GELU_A * (1 + 3 * _GELU_B * g * g)
    dt = s["dh"].dtype
    dg, du = (dh * u * da).to(dt), (dh * a).to(dt)
    dx = dg.float() @ _values(s["gate"]) + du.float() @ _values(s["up"])
    return {"dg": dg, "du": du, "dx": dx.to(dt)}


_PLAIN = {"quantize": _p_quantize, "gemm": _p_gemm, "gemm_bwd": _p_gemm_bwd, "gated": _p_gated,
          "gated_bwd": _p_gated_bwd}


# ------------------------------------------------------------------------------------
# what a pass cannot do without
# ------------------------------------------------------------------------------------

_SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def work(case):
    c = case
    kind, t, k, b = c["kind"], c["t"], c["k"], _SIZE[c["type"]]
    if kind == "quantize":
        return {"bytes": t * k * 2 * b + t * k * 17 // 32, "flops": 2 * t * k}
    n = c["n"]
    if kind == "gemm":
        return {"bytes": (t + n) * k * 17 // 32 + t * n * b, "flops": 2 * t * n * k}
    if kind == "gemm_bwd":
        return {"bytes": n * k * 17 // 32 + t * (n + k) * b, "flops": 2 * t * n * k}
    if kind == "gated":
        io = t * n * (b * (3 if c["save"] else 1) + (8 if c["add"] else 0))
        return {"bytes": (t + 2 * n) * k * 17 // 32 + io, "flops": 4 * t * n * k}
    return {"bytes": 2 * n * k * 17 // 32 + t * (5 * n + k) * b, "flops": 4 * t * n * k}


# ------------------------------------------------------------------------------------
# results in 64 bits
# ------------------------------------------------------------------------------------

def exact(case, seed):
    s = _DRAW[case["kind"]](case, _gen(seed))
    return _EXACT[case["kind"]](case, s)


def _x_dequantized(q):
    """(-1)^s 2^(E-127) times (1 + m/2) 2^(e-1), or m/2 where e = 0; in 64 bits, a block of 32 at a time."""
    codes, scales = q
    rows, nb = scales.shape
    out = torch.empty(rows, nb, 2, 16, device="cuda", dtype=torch.float64)
    for half in (0, 1):
        c = (codes.reshape(rows, nb, 16) >> (4 * half)) & 15
        e, m = ((c >> 1) & 3).double(), (c & 1).double()
        mag = torch.where(e == 0, 0.5 * m, (1 + 0.5 * m) * 2.0 ** (e - 1))
        out[:, :, half] = torch.where(c >= 8, -mag, mag) * 2.0 ** (scales.double() - 127)[..., None]
    return out.reshape(rows, nb * 32)


def _x_quantize(c, s):
    """Each element goes to the nearest of the 16 values times its block's scale, of two equally near ones to the
    one of even mantissa; magnitudes past the largest go to it."""
    x = s["x"].double().reshape(-1, 32)
    top = x.abs().amax(dim=1, keepdim=True)
    e = torch.floor(torch.log2(torch.where(top > 0, top, 1.0)))
    e = e + (2.0 ** (e + 1) <= top).double() - (2.0 ** e > top).double()  # log2 may round over a power of two
    scale = 2.0 ** (e - 2)
    if c["noclip"]:
        scale = torch.where(top > 6 * scale, 2 * scale, scale)
    r = (x.abs() / scale).clamp(max=6.0)
    step = torch.where(r < 2, 0.5, torch.where(r < 4, 1.0, 2.0))
    v = torch.round(r / step) * step * scale  # (torch.round: halves to even)
    return {"codes": None, "scales": None, "values": torch.where(top > 0, torch.copysign(v, x), x).reshape(s["x"].shape)}


def _x_gemm(c, s):
    return {"y": _x_dequantized(s["xq"]) @ _x_dequantized(s["w"]).t()}


def _x_gemm_bwd(c, s):
    return {"dx": s["dy"].double() @ _x_dequantized(s["w"])}


def _x_act(c, g):
    if c["act"] == "silu":
        return g * torch.sigmoid(g)
    return 0.5 * g * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)))


def _x_gated(c, s):
    x = _x_dequantized(s["xq"])
    g, u = x @ _x_dequantized(s["gate"]).t(), x @ _x_dequantized(s["up"]).t()
    if c["add"]:
        g, u = g + s["g_add"].double(), u + s["u_add"].double()
    o = {"h": _x_act(c, g) * u}
    if c["save"]:
        o["g"], o["u"] = g, u
    return o


def _x_gated_bwd(c, s):
    """dg and du by automatic differentiation of act(g) u; dx of the two rounded to the type, as they are returned."""
    g, u = s["g"].double().requires_grad_(True), s["u"].double().requires_grad_(True)
    dg, du = torch.autograd.grad(_x_act(c, g) * u, (g, u), s["dh"].double())
    dt = s["dh"].dtype
    dx = dg.to(dt).double() @ _x_dequantized(s["gate"]) + du.to(dt).double() @ _x_dequantized(s["up"])
    return {"dg": dg, "du": du, "dx": dx}


_EXACT = {"quantize": _x_quantize, "gemm": _x_gemm, "gemm_bwd": _x_gemm_bwd, "gated": _x_gated,
          "gated_bwd": _x_gated_bwd}
