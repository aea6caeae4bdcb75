"""Performance cases of the operators behind the framework's two projections:
the gated feed-forward and the norm and rotation of queries and keys.

Five kinds of call, with ``own`` through the package's public Python entry
points, without it in elementary torch operations:

* ``gated``    MXNorm, gate and up projections, activation and product (bf16 H;
  a training step also keeps the projections for its backward pass);
* ``ffn``      the same with H in MX codes, and the down projection that takes
  them;
* ``gatedbwd`` the gradients of ``gated``: x, the gain, the weight;
* ``qk``       the norm of every query and key head and its rotation, read from
  the fused projection's output;
* ``qkbwd``    its gradients, into the fused projection's gradient.

Activations are N(0, 1) with 1% outlier channels at 20 times that, weights
0.02 N(0, 1), gains 1 + 0.1 N(0, 1), output gradients 0.01 N(0, 1).
"""
import math

import torch

own = False

DEV = "cuda"
EPS = 1e-6
# MXNorm's RMS coefficient of 32-element blocks, by the exponent of the mean
COEF = {1: 0.4261, 2: 0.4185}


def listed():
    return [
        # one token through the gate and up projections of an 8B model: the
        # smallest feed-forward call, the weights' bytes alone
        dict(name="gated_decode1", op="gated", elem="e4m3", act="silu", T=1, d=4096, F=14336, p=2, train=False),
        # a ragged prefill chunk of a small model with the other activation
        dict(name="gated_ragged", op="gated", elem="e4m3", act="gelu_tanh", T=1000, d=2048, F=4096, p=1, train=False),
        # a 16k-token training step in 4 bits, projections kept: the largest forward
        dict(name="gated_train16k_fp4", op="gated", elem="e2m1", act="silu", T=16384, d=4096, F=14336, p=2, train=True),
        # one decoding step of 61 sequences through the whole feed-forward, 4-bit weights
        dict(name="ffn_decode61_fp4", op="ffn", elem="e2m1", act="silu", T=61, d=4096, F=14336, p=2),
        # prefill of 8192 tokens through the whole feed-forward
        dict(name="ffn_prefill8k", op="ffn", elem="e4m3", act="silu", T=8192, d=4096, F=14336, p=2),
        # one 1024-token step of a 125M-parameter model: launches and latency
        dict(name="gatedbwd_125m", op="gatedbwd", elem="e4m3", act="gelu_tanh", T=1024, d=768, F=2048),
        # a batch whose token count is no multiple of anything, 4 bits
        dict(name="gatedbwd_ragged_fp4", op="gatedbwd", elem="e2m1", act="silu", T=1999, d=2048, F=4096),
        # backward of an 8B model's feed-forward at 8k tokens: the largest call
        dict(name="gatedbwd_8k", op="gatedbwd", elem="e4m3", act="silu", T=8192, d=4096, F=14336),
        # one decoding step of 16 sequences at far positions: latency
        dict(name="qk_decode16", op="qk", T=16, Hq=32, Hk=8, D=128, R=128, interleaved=False, far=1 << 20),
        # a 32k-token training step of an 8B model: bandwidth
        dict(name="qk_train32k", op="qk", T=32768, Hq=32, Hk=8, D=128, R=128, interleaved=False, far=8192),
        # a small model's odd batch, half of each head rotated in adjacent pairs
        dict(name="qkbwd_ragged", op="qkbwd", T=1999, Hq=12, Hk=4, D=64, R=32, interleaved=True, far=2048),
        # the gradients of the 32k-token step
        dict(name="qkbwd_train32k", op="qkbwd", T=32768, Hq=32, Hk=8, D=128, R=128, interleaved=False, far=8192),
    ]


def _log(rng, lo, hi, mult=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(mult, int(round(v / mult)) * mult)


def draw(rng):
    """One more case: a kind by its weight, sizes log-uniform over the range."""
    op = rng.choice(["gated", "gated", "ffn", "ffn", "gatedbwd", "gatedbwd", "qk", "qkbwd"])
    if op in ("qk", "qkbwd"):
        D = rng.choice([64, 80, 96, 128, 128, 256])
        Hk = rng.choice([1, 2, 4, 8, 8])
        Hq = Hk * rng.choice([1, 2, 3, 4, 8])
        R = rng.choice([D, D, D // 2 // 16 * 16])
        most = 32768 * 40 * 128 // ((Hq + Hk) * D)
        T = rng.choice([_log(rng, 1, 512), _log(rng, 512, 65536)])
        return dict(op=op, T=min(T, most), Hq=Hq, Hk=Hk, D=D, R=R, interleaved=rng.choice([False, False, True]),
                    far=_log(rng, 1024, 1 << 20))
    elem = rng.choice(["e4m3", "e4m3", "e2m1"])
    act = rng.choice(["silu", "silu", "gelu_tanh"])
    step = 128 if elem == "e4m3" else 256  # contraction lengths the products take
    d = _log(rng, 512, 6144, step)
    if op == "gatedbwd":
        F = _log(rng, 512, 16384, step)
        most = 8192 * 14336 * 4096 // (d * F)
        T = rng.choice([_log(rng, 32, 1024), _log(rng, 1024, 16384)])
        return dict(op=op, elem=elem, act=act, T=min(T, most), d=d, F=F)
    F = _log(rng, 512, 16384, 16 if op == "gated" else step)
    # the down projection's work is half the others'
    most = 8192 * 14336 * 4096 // (d * F)
    T = rng.choice([_log(rng, 1, 256), _log(rng, 256, 16384)])
    case = dict(op=op, elem=elem, act=act, T=min(T, most), d=d, F=F, p=rng.choice([1, 2, 2]))
    if op == "gated":
        case["train"] = rng.choice([False, True])
    return case


# ------------------------------------------------------------------ inputs --

def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.bfloat16)


def _activations(g, T, d):
    x = _normal(g, T, d)
    ch = torch.randperm(d, generator=g, device=DEV)[:max(1, d // 100)]
    x[:, ch] *= 20
    return x


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    c, op, T = dict(case), case["op"], case["T"]
    if op in ("qk", "qkbwd"):
        Hq, Hk, D, R = c["Hq"], c["Hk"], c["D"], c["R"]
        # the fused projection's output: queries, keys, values of each token
        qkv = _normal(g, T, (Hq + 2 * Hk) * D) * 3
        c["q"] = qkv[:, :Hq * D].view(T, Hq, D)
        c["k"] = qkv[:, Hq * D:(Hq + Hk) * D].view(T, Hk, D)
        c["qg"], c["kg"] = 1 + 0.1 * _normal(g, D), 1 + 0.1 * _normal(g, D)
        # packed sequences of many lengths (one token each where T is small)
        far = torch.randint(0, c["far"], (T,), generator=g, device=DEV)
        c["pos"] = far if T <= 512 else (torch.arange(T, device=DEV) + int(far[0])) % c["far"]
        c["inv_freq"] = (500000.0 ** (-torch.arange(0, R, 2, device=DEV, dtype=torch.float64) / max(R, 1))).float()
        if op == "qkbwd":
            c["gq"], c["gk"] = 0.01 * _normal(g, T, Hq, D), 0.01 * _normal(g, T, Hk, D)
            # where the gradient of the projection's output is collected
            gqkv = torch.zeros_like(qkv)
            c["oq"] = gqkv[:, :Hq * D].view(T, Hq, D)
            c["ok"] = gqkv[:, Hq * D:(Hq + Hk) * D].view(T, Hk, D)
        return c
    d, F = c["d"], c["F"]
    c["x"] = _activations(g, T, d)
    c["gamma"] = 1 + 0.1 * _normal(g, d)
    w = 0.02 * _normal(g, 2 * F, d)
    if op == "gatedbwd":
        c["w"] = w
        c["gh"] = 0.01 * _normal(g, T, F)
        # what the forward of this step kept
        c["gu"] = _normal(g, T, 2 * F)
        c["rho"] = _rho(c["x"], 2)
        return c
    # weights that a serving program casts once
    c["wc"], c["ws"] = _encode(w.float() * c["gamma"].float(), c["elem"])
    if op == "ffn":
        c["dc"], c["ds"] = _encode((0.02 * _normal(g, d, F)).float(), c["elem"])
    return c


# -------------------------------------------------- the operators, plainly --

def _pow2f(e):
    """2^e in float32 for integers e from -126 to 127."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _encode(t, elem):
    """MX encoding of float32 rows along the last axis: (codes, scales), blocks
    of 32, power-of-two scales rounded up so that nothing saturates."""
    n, d = t.shape
    v = t.reshape(n, d // 32, 32)
    a = v.abs().amax(-1).view(torch.int32)
    e = ((a + 0x1FFFFF) >> 23) - 8 if elem == "e4m3" else ((a + 0x3FFFFF) >> 23) - 2
    e = e.clamp(min=1)
    q = (v * _pow2f(127 - e)[..., None]).reshape(n, d)
    if elem == "e4m3":
        codes = q.to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        m = q.abs()
        m = torch.where(m < 2, torch.round(2 * m), torch.where(m < 4, torch.round(m) + 2, torch.round(m / 2) + 4))
        m = (m.to(torch.uint8) | (q < 0).to(torch.uint8) << 3).reshape(n, d // 2, 2)
        codes = m[..., 0] | m[..., 1] << 4
    return codes, e.to(torch.uint8)


def _decode(codes, scales, elem):
    """Float32 values of MX codes and scales."""
    if elem == "e4m3":
        v = codes.view(torch.float8_e4m3fn).float()
    else:
        n = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()
        values = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
        v = values[n]
    n, d = v.shape
    return (v.reshape(n, d // 32, 32) * _pow2f(scales.int() - 127)[..., None]).reshape(n, d)


def _rho(x, p):
    """MXNorm's inverse RMS estimate, in 64 bits and rounded once."""
    T, d = x.shape
    m = x.reshape(T, d // 32, 32).abs().amax(-1).double()
    mean = m.mean(-1) if p == 1 else (m * m).mean(-1).sqrt()
    coef = float(torch.tensor(COEF[p], dtype=torch.float32))
    eps = float(torch.tensor(EPS, dtype=torch.float32))
    return (1 / ((coef * mean) ** 2 + eps).sqrt()).float()


def _gate(g, act):
    """(sigma(z(g)), dz/dg) of the activation g sigma(z(g))."""
    if act == "silu":
        z, dz = g, torch.ones_like(g)
    else:
        c = 2 * math.sqrt(2 / math.pi)
        z, dz = c * (g + 0.044715 * g * g * g), c * (1 + 3 * 0.044715 * g * g)
    return 1 / (1 + torch.exp(-z)), dz


def _gated(s):
    """(G U, rho, float32 H) of the norm, the two projections and the gate."""
    rho = _rho(s["x"], s["p"])
    z = _decode(*_encode(s["x"].float() * rho[:, None], s["elem"]), s["elem"])
    gu = z @ _decode(s["wc"], s["ws"], s["elem"]).t()
    g, u = gu.split(s["F"], 1)
    return gu, rho, g * _gate(g, s["act"])[0] * u


def _rotation(s):
    """cos and sin of every token's angles, float32 [T, 1, R/2]."""
    a = (s["pos"].double()[:, None] * s["inv_freq"].double())[:, None]
    return torch.cos(a).float(), torch.sin(a).float()


def _pairs(y, R, interleaved):
    """The two halves of each rotated pair, and the part that is not rotated."""
    r = y[..., :R]
    if interleaved:
        return r[..., 0::2], r[..., 1::2], y[..., R:]
    return r[..., :R // 2], r[..., R // 2:], y[..., R:]


def _rejoin(a, b, rest, interleaved):
    r = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((r, rest), -1)


def _head(s, rot, x, gamma):
    x = x.float()
    r = 1 / (x.square().mean(-1, keepdim=True) + EPS).sqrt()
    a, b, rest = _pairs(x * r * gamma.float(), s["R"], s["interleaved"])
    y = _rejoin(a * rot[0] - b * rot[1], b * rot[0] + a * rot[1], rest, s["interleaved"])
    return y.bfloat16()


def _head_gradient(s, rot, gy, x, gamma):
    x, gamma = x.float(), gamma.float()
    r = 1 / (x.square().mean(-1, keepdim=True) + EPS).sqrt()
    a, b, rest = _pairs(gy.float(), s["R"], s["interleaved"])
    gn = _rejoin(a * rot[0] + b * rot[1], b * rot[0] - a * rot[1], rest, s["interleaved"])
    u = (gn * gamma * x).sum(-1, keepdim=True)
    gx = r * gamma * gn - r * r * r * u / s["D"] * x
    return gx.bfloat16(), (r * x * gn).sum((0, 1), dtype=torch.float64).float()


def _plain(s):
    op = s["op"]
    if op == "gated":
        gu, rho, h = _gated(s)
        return (h.bfloat16(), gu.bfloat16(), rho) if s["train"] else h.bfloat16()
    if op == "ffn":
        h = _decode(*_encode(_gated(s)[2], s["elem"]), s["elem"])
        return (h @ _decode(s["dc"], s["ds"], s["elem"]).t()).bfloat16()
    if op == "qk":
        rot = _rotation(s)
        return _head(s, rot, s["q"], s["qg"]), _head(s, rot, s["k"], s["kg"])
    if op == "qkbwd":
        rot = _rotation(s)
        gq, gqg = _head_gradient(s, rot, s["gq"], s["q"], s["qg"])
        gk, gkg = _head_gradient(s, rot, s["gk"], s["k"], s["kg"])
        s["oq"].copy_(gq)
        s["ok"].copy_(gk)
        return s["oq"], s["ok"], gqg, gkg
    elem, T, d = s["elem"], s["T"], s["d"]
    g, u = s["gu"].float().split(s["F"], 1)
    gh, x, rho, gamma = s["gh"].float(), s["x"].float(), s["rho"][:, None], s["gamma"].float()
    sg, dz = _gate(g, s["act"])
    # the gradients of the projections: bf16, as the casts take them
    gp = torch.cat((gh * u * (sg + g * sg * (1 - sg) * dz), gh * g * sg), 1).bfloat16().float()
    wt = _decode(*_encode(s["w"].t().float().contiguous(), elem), elem)
    gz = (_decode(*_encode(gp, elem), elem) @ wt.t()).bfloat16().float()
    un = (gz * gamma * x).sum(-1, keepdim=True)
    gx = rho * gz * gamma - rho * rho * rho * un / d * x
    gg = (rho * x * gz).sum(0, dtype=torch.float64)
    # the weight's gradient contracts over tokens: whole blocks of them
    pad = torch.zeros(-T % 32, 1, device=DEV)
    gpt = torch.cat((gp, pad.expand(-1, 2 * s["F"]))).t().contiguous()
    xt = torch.cat((x * rho, pad.expand(-1, d))).t().contiguous()
    gw = _decode(*_encode(gpt, elem), elem) @ _decode(*_encode(xt, elem), elem).t()
    return gx.bfloat16(), gg.bfloat16(), (gw * gamma).bfloat16()


def run(s):
    if not own:
        return _plain(s)
    from paper_2603_13180_amd import mxnorm
    op = s["op"]
    if op == "gated":
        h, gu, rho = mxnorm.mxnorm_gated_fwd(s["x"], s["wc"], s["ws"], elem=s["elem"], p=s["p"], act=s["act"],
                                             save_gu=s["train"], want_rho=s["train"])
        return (h, gu, rho) if s["train"] else h
    if op == "ffn":
        (hc, hs), _, _ = mxnorm.mxnorm_gated_fwd(s["x"], s["wc"], s["ws"], elem=s["elem"], p=s["p"], act=s["act"],
                                                 out_dtype=torch.uint8, want_rho=False)
        return mxnorm.mx_matmul_fwd(hc, hs, s["dc"], s["ds"], s["F"], elem=s["elem"], out_dtype=torch.bfloat16)
    if op == "gatedbwd":
        return mxnorm.mxnorm_gated_bwd(s["gh"], s["gu"], s["x"], s["rho"], s["gamma"], s["w"], elem=s["elem"],
                                       act=s["act"], grad_dtype=torch.bfloat16)
    kw = dict(rotary=s["R"], interleaved=s["interleaved"], eps=EPS)
    if op == "qk":
        return mxnorm.qk_norm_rope_fwd(s["q"], s["k"], s["qg"], s["kg"], s["pos"], s["inv_freq"], **kw)
    return mxnorm.qk_norm_rope_bwd(s["gq"], s["gk"], s["q"], s["k"], s["qg"], s["kg"], s["pos"], s["inv_freq"],
                                   grad_q=s["oq"], grad_k=s["ok"], **kw)


# -------------------------------------------------------------------- work --

def _codes(n, elem):
    return n + n // 32 if elem == "e4m3" else n // 2 + n // 32


def work(case):
    op, T = case["op"], case["T"]
    if op in ("qk", "qkbwd"):
        n, D = T * (case["Hq"] + case["Hk"]) * case["D"], case["D"]
        small = 4 * D + 8 * T + 2 * case["R"]
        if op == "qk":
            return {"bytes": 4 * n + small, "flops": 8 * n}
        return {"bytes": 6 * n + small + 8 * D, "flops": 16 * n}
    d, F, elem = case["d"], case["F"], case["elem"]
    if op == "gatedbwd":
        return {"bytes": 2 * T * F + 4 * T * F + 2 * T * d + 4 * T + 4 * F * d + 2 * d + 2 * T * d + 2 * d + 4 * F * d,
                "flops": 8 * T * F * d}
    n = 2 * T * d + _codes(2 * F * d, elem)
    if op == "ffn":
        return {"bytes": n + _codes(F * d, elem) + 2 * T * d, "flops": 6 * T * F * d}
    return {"bytes": n + 2 * T * F + (4 * T * F + 4 * T if case["train"] else 0), "flops": 4 * T * F * d}


# ------------------------------------------------------- the same in 64 bits --

def _exact_pow2(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _mx(t, elem):
    """Values (float64) of the MX encoding of rows t along the last axis, from
    the formats' definition: the smallest power of two under which the block's
    largest magnitude is in range, then the nearest multiple of each value's
    step, ties to even."""
    n, d = t.shape
    big, man, low = (448.0, 3, -6) if elem == "e4m3" else (6.0, 1, 0)
    out = torch.empty(n, d, dtype=torch.float64, device=t.device)
    rows = max(1, (1 << 26) // d)
    for r in range(0, n, rows):
        v = t[r:r + rows].double().reshape(-1, d // 32, 32)
        e = torch.frexp(v.abs().amax(-1, keepdim=True) / big)
        ex = torch.where(e.mantissa == 0.5, e.exponent - 1, e.exponent).clamp(min=-126)
        q = v * _exact_pow2(-ex)
        step = _exact_pow2((torch.frexp(q).exponent - 1).clamp(min=low) - man)
        out[r:r + rows] = (torch.round(q / step) * step * _exact_pow2(ex)).reshape(-1, d)
    return out


def _values(codes, scales, elem):
    """Values (float64) of given codes, bit field by bit field."""
    if elem == "e4m3":
        c, man, bias = codes.int(), 3, 7
    else:
        c, man, bias = torch.stack((codes & 15, codes >> 4), 2).reshape(codes.shape[0], -1).int(), 1, 1
    field = c & ((8 << 4) - 1 if elem == "e4m3" else 7)
    E, M = field >> man, (field & ((1 << man) - 1)).double() / (1 << man)
    v = torch.where(E == 0, M * 2.0 ** (1 - bias), (1 + M) * _exact_pow2(E - bias))
    v = torch.where(c >> (7 if elem == "e4m3" else 3) == 1, -v, v)
    return v * _exact_pow2(scales.int() - 127).repeat_interleave(32, 1)


def _exact_act(g, act):
    """(act(g), act'(g)) in 64 bits, through the hyperbolic tangent."""
    if act == "silu":
        t = torch.tanh(g / 2)
        return g * (1 + t) / 2, (1 + t) / 2 + g * (1 - t * t) / 4
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g ** 3))
    return g * (1 + t) / 2, (1 + t) / 2 + g / 2 * (1 - t * t) * c * (1 + 3 * 0.044715 * g ** 2)


def _exact_heads(s, x, gamma, gy=None):
    T, H, D = x.shape
    R, x, gamma = s["R"], x.double(), gamma.double()
    # the rotation as a product of complex numbers
    a = s["pos"].double()[:, None, None] * s["inv_freq"].double()
    turn = torch.polar(torch.ones_like(a), a)
    i = torch.arange(R, device=DEV)
    first, second = (i[0::2], i[1::2]) if s["interleaved"] else (i[:R // 2], i[R // 2:])
    ms = x.square().sum(-1, keepdim=True) / D + EPS
    y = (x / ms.sqrt() * gamma if gy is None else gy.double()).clone()
    c = torch.complex(y[..., first], y[..., second]) * (turn if gy is None else turn.conj())
    y[..., first], y[..., second] = c.real, c.imag
    if gy is None:
        return y
    xn = x / ms.sqrt()
    v = y * gamma
    return (v - xn * (v * xn).mean(-1, keepdim=True)) / ms.sqrt(), (xn * y).sum((0, 1))


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "qk":
        return _exact_heads(s, s["q"], s["qg"]), _exact_heads(s, s["k"], s["kg"])
    if op == "qkbwd":
        gq, gqg = _exact_heads(s, s["q"], s["qg"], s["gq"])
        gk, gkg = _exact_heads(s, s["k"], s["kg"], s["gk"])
        return gq, gk, gqg, gkg
    elem, d, F, T = case["elem"], case["d"], case["F"], case["T"]
    x = s["x"].double()
    if op == "gatedbwd":
        rho, gamma = s["rho"].double(), s["gamma"].double()
        a, da = _exact_act(s["gu"][:, :F].double(), case["act"])
        gh = s["gh"].double()
        gp = torch.cat((gh * s["gu"][:, F:].double() * da, gh * a), 1).bfloat16()
        gz = _mx(gp, elem) @ _mx(s["w"].t().contiguous(), elem).t().contiguous()
        v = gz * gamma
        gx = rho[:, None] * v - (rho ** 3 / d * (v * x).sum(-1))[:, None] * x
        gg = (rho[:, None] * x * gz).sum(0)
        rows = -(-T // 32) * 32
        gpt = torch.zeros(2 * F, rows, dtype=torch.bfloat16, device=DEV)
        gpt[:, :T] = gp.t()
        xt = torch.zeros(d, rows, dtype=torch.float32, device=DEV)
        xt[:, :T] = (s["x"].float() * s["rho"][:, None]).t()
        return gx, gg, _mx(gpt, elem) @ _mx(xt, elem).t().contiguous() * gamma
    m = x.reshape(T, d // 32, 32).abs().amax(-1)
    rms = float(torch.tensor(COEF[case["p"]], dtype=torch.float32)) * (m ** case["p"]).mean(-1) ** (1 / case["p"])
    rho = (rms ** 2 + float(torch.tensor(EPS, dtype=torch.float32))) ** -0.5
    gu = _mx(s["x"].float() * rho.float()[:, None], elem) @ _values(s["wc"], s["ws"], elem).t().contiguous()
    h = _exact_act(gu[:, :F], case["act"])[0] * gu[:, F:]
    if op == "ffn":
        return _mx(h, elem) @ _values(s["dc"], s["ds"], elem).t().contiguous()
    return (h, gu, rho) if case["train"] else h
