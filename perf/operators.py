"""The steps of a decoder layer that stand beside its FP8 linears, each through
one public call: what is measured, their plain form and their exact results.

Kinds of case
  qk              RMSNorm of each query and key head and the position rotation,
                  in one pass over views of the qkv output
  qk_backward     its gradients: dq, dk and the gains'
  linear          a linear with bias, activation and residual in its epilogue:
                  z = x w^T + bias, y = act(z) + residual
  act_backward    the epilogue's backward: dz = dy act'(z), dbias = sum dz, dz
                  in BF16 or as the two FP8 copies that Dgrad and Wgrad read
  gated           the gated feed-forward's two projections, activation and
                  product: h = act(x wg^T) * (x wu^T), h in BF16 or as the two FP8
                  copies that the down projection and its Wgrad read
  gated_backward  dgate = dh up act'(gate), dup = dh act(gate), in BF16 or as
                  FP8 copies

Operands of the products are BF16 ("bf16"), FP8 with a power-of-two scale for
each 1x128 group of activations and 128x128 block of weights ("block"), or FP8
with one scale ("tensor").  What an FP8 copy is: the values rounded to BF16, the
smallest power of two 2^k with amax <= fmt_max 2^k for each group, and the
values times 2^-k rounded to FP8.  Codes are returned as the float8 numbers that
they are, scales as the E8M0 numbers that they are.
"""
import math

import torch

own = False

DEV = "cuda"
EPS = 1e-6
ROPE_BASE = 1e6
ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh")
F8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
FMT_MAX_EXP = {"e4m3": 9, "e5m2": 16}  # fmt_max = 0.875 * 2^this
MAX_FLOPS = 4 * 32768 * 8960 * 1536  # of the largest listed case


def listed():
    return [
        # the Qwen3-1.7B attention input at the paper's micro-batch of 2 x 4096 tokens
        dict(name="qk_m8192", kind="qk", t=8192, hq=16, hkv=8, d=128, rot=128, inter=False, seqs=2, pad=0),
        # one token, as a model that generates calls it: nothing but latency
        dict(name="qk_token", kind="qk", t=1, hq=16, hkv=8, d=128, rot=128, inter=False, seqs=1, pad=0),
        # its backward in training
        dict(name="qk_backward_m8192", kind="qk_backward", t=8192, hq=16, hkv=8, d=128, rot=128, inter=False, seqs=2, pad=0),
        # packed sequences of odd lengths and padding rows behind them, half of each head rotated in neighbouring pairs
        dict(name="qk_backward_ragged", kind="qk_backward", t=5003, hq=12, hkv=2, d=128, rot=64, inter=True, seqs=7, pad=37),
        # the Qwen3-1.7B down projection, added to the residual stream
        dict(name="linear_down_m8192", kind="linear", ops="block", m=8192, n=2048, k=6144, bias=False, act="none",
             residual=True, z=False),
        # the down projection of one token in BF16: bound by the weights
        dict(name="linear_down_token", kind="linear", ops="bf16", m=1, n=1536, k=8960, bias=False, act="none",
             residual=True, z=False),
        # an ungated MLP's first linear in training, Qwen2-1.5B widths
        dict(name="act_backward_m8192", kind="act_backward", ops="block", fmt="e4m3", m=8192, n=8960, act="gelu_tanh", dbias=True),
        # the gradient of a linear's bias and activation in BF16, tokens of a ragged batch
        dict(name="act_backward_ragged", kind="act_backward", ops="bf16", fmt="e4m3", m=1337, n=1536, act="silu", dbias=True),
        # the Qwen2-1.5B MLP in training: 32768 tokens, gate and up kept for the backward
        dict(name="gated_m32768", kind="gated", ops="block", fmt="e4m3", m=32768, f=8960, k=1536, act="silu", keep=True),
        # the same MLP on one token in BF16
        dict(name="gated_token", kind="gated", ops="bf16", fmt="e4m3", m=1, f=8960, k=1536, act="silu", keep=False),
        # the Qwen3-1.7B MLP's backward at the paper's micro-batch
        dict(name="gated_backward_m8192", kind="gated_backward", ops="block", fmt="e4m3", m=8192, f=6144, act="silu"),
        # a BF16 model's on a ragged batch
        dict(name="gated_backward_ragged", kind="gated_backward", ops="bf16", fmt="e4m3", m=777, f=6144, act="gelu"),
    ]


def _log(rng, lo, hi, step):
    """A multiple of step between lo and hi, even over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step))


def draw(rng):
    kind = rng.choice(["qk", "qk_backward", "linear", "act_backward", "gated", "gated_backward"])
    if kind.startswith("qk"):
        d = rng.choice([64, 80, 96, 128, 192, 256])
        t = _log(rng, 1, 16384, 1)
        hkv = rng.choice([1, 2, 4, 8])
        return dict(kind=kind, t=t, hq=hkv * rng.choice([1, 2, 4, 6]), hkv=hkv, d=d,
                    rot=rng.choice([d, d // 2 // 16 * 16]), inter=rng.random() < 0.3, seqs=rng.randint(1, max(1, min(8, t))),
                    pad=rng.choice([0, 0, t // 9]))
    ops = rng.choice(["block", "block", "bf16"])
    fmt = rng.choice(["e4m3", "e4m3", "e5m2"])
    step_m, step = (128, 128) if ops == "block" else (1, 8)
    if kind == "linear":
        if rng.random() < 0.25:
            ops, step_m, step = "tensor", 16, 16
        n, k = _log(rng, 256, 9216, step), _log(rng, 256, 9216, step)
        m = _log(rng, step_m, min(32768 if ops != "bf16" else 8192, MAX_FLOPS // (2 * n * k) // step_m * step_m), step_m)
        act = rng.choice(ACTS)
        return dict(kind=kind, ops=ops, m=m, n=n, k=k, bias=rng.random() < 0.6, act=act, residual=rng.random() < 0.6,
                    z=act != "none" and rng.random() < 0.5)
    if kind == "act_backward":
        return dict(kind=kind, ops=ops, fmt=fmt, m=_log(rng, step_m, 16384, step_m), n=_log(rng, 256, 9216, step),
                    act=rng.choice(ACTS), dbias=rng.random() < 0.7)
    act = rng.choice(("silu", "silu", "gelu", "gelu_tanh", "relu"))
    if kind == "gated":
        m = _log(rng, step_m, 16384 if ops == "block" else 4096, step_m)
        return dict(kind=kind, ops=ops, fmt=fmt, m=m, f=_log(rng, 256, 9216, step), k=_log(rng, 256, 4096, step), act=act,
                    keep=rng.random() < 0.6)
    return dict(kind=kind, ops=ops, fmt=fmt, m=_log(rng, step_m, 16384, step_m), f=_log(rng, 256, 9216, step), act=act)


# ------------------------------------------------------------- FP8 copies
def _act_groups(x, f8, fmt_exp):
    """x [R, C] (BF16 values in 32 or 64 bits): x / 2^k in 1x128 groups, and k + 127 [R, C / 128]."""
    r, c = x.shape
    g = x.view(r, c // 128, 128)
    amax = g.abs().amax(-1)
    m, e = torch.frexp(amax)
    k = torch.where(amax > 0, e - fmt_exp + (m > 0.875), torch.zeros_like(e)).clamp(-127, 127)
    return torch.ldexp(g, -k[..., None]).view(r, c), (k + 127).to(torch.uint8)


def _weight_blocks(w, fmt_exp):
    r, c = w.shape
    amax = w.view(r // 128, 128, c // 128, 128).abs().amax((1, 3))
    m, e = torch.frexp(amax)
    k = torch.where(amax > 0, e - fmt_exp + (m > 0.875), torch.zeros_like(e))
    k = k.repeat_interleave(128, 0)
    return torch.ldexp(w.view(r, c // 128, 128), -k[..., None]).view(r, c), (k + 127).to(torch.uint8)


def _pack_scales(g):
    """E8M0 exponents [R, KB] in the library's layout [R/128, ceil(KB/4), 512] (include/puro_fp8.h)."""
    r, kb = g.shape
    kg = (kb + 3) // 4
    full = torch.full((r, kg * 4), 127, dtype=torch.uint8, device=g.device)
    full[:, :kb] = g
    return full.view(r // 128, 4, 32, kg, 4).permute(0, 3, 2, 1, 4).reshape(r // 128, kg, 512)


def _unpack_scales(s, kb):
    rb, kg, _ = s.shape
    return s.view(rb, kg, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(rb * 128, kg * 4)[:, :kb]


def _copies(x, fmt, both):
    """The FP8 copies of x (32 bits): codes, scales, and both of the transpose."""
    x = x.to(torch.bfloat16).float()
    out = {}
    for name, v in (("q", x), ("q_t", x.t().contiguous())) if both else (("q", x),):
        scaled, g = _act_groups(v, F8[fmt], FMT_MAX_EXP[fmt])
        out[name] = scaled.to(F8[fmt])
        out[name + "_scale"] = _pack_scales(g).view(torch.float8_e8m0fnu)
    return out


def _exact_copies(x, fmt, both):
    """What the copies' numbers stand for in 64 bits: each value over its group's power of two, not rounded, and that power."""
    out = {}
    for name, v in (("q", x), ("q_t", x.t().contiguous())) if both else (("q", x),):
        _, g = _act_groups(v.to(torch.bfloat16).double(), F8[fmt], FMT_MAX_EXP[fmt])
        r, c = v.shape
        k = g.int() - 127
        out[name] = torch.ldexp(v.view(r, c // 128, 128), -k[..., None]).view(r, c)
        out[name + "_scale"] = torch.exp2((_pack_scales(g).int() - 127).double())
    return out


def _operand(v, ops, weight):
    """An operand of a product as a program holds it: BF16 values, or FP8 codes and scales."""
    if ops == "bf16":
        return {"x": v}
    if ops == "tensor":
        scale = 448.0 / v.float().abs().amax()
        return {"codes": (v.float() * scale).to(F8["e4m3"]).view(torch.uint8), "scale": (1.0 / scale).reshape(1)}
    scaled, g = _weight_blocks(v.float(), 9) if weight else _act_groups(v.float(), F8["e4m3"], 9)
    return {"codes": scaled.to(F8["e4m3"]).view(torch.uint8), "scale": _pack_scales(g)}


def _values(o, ops, dtype):
    """The numbers that an operand stands for."""
    if ops == "bf16":
        return o["x"].to(dtype)
    v = o["codes"].view(F8["e4m3"]).to(dtype)
    if ops == "tensor":
        return v * o["scale"].to(dtype)
    r, c = v.shape
    k = _unpack_scales(o["scale"], c // 128).int() - 127
    return torch.ldexp(v.view(r, c // 128, 128), k[..., None]).view(r, c)


# ------------------------------------------------------------- activations
def _act(z, act):
    if act == "none":
        return z
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * torch.erfc(-z * math.sqrt(0.5))
    return z / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))  # 0.5 z (1 + tanh(u)) = z sigmoid(2 u)


def _act_slope(z, act):
    if act == "none":
        return torch.ones_like(z)
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * torch.erfc(-z * math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    c = 2 * math.sqrt(2 / math.pi)
    u, du = (z, 1.0) if act == "silu" else (c * (z + 0.044715 * z ** 3), c * (1 + 3 * 0.044715 * z * z))
    s, r = 1 / (1 + torch.exp(-u)), 1 / (1 + torch.exp(u))
    return s + z * s * r * du


# ------------------------------------------------------------- inputs
def _gen(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed(64 * seed + stream)
    return g


def _normal(shape, std, seed, stream):
    return torch.randn(shape, generator=_gen(seed, stream), device=DEV).mul_(std).to(torch.bfloat16)


def _normed(shape, seed, stream):
    """Rows as a norm with a few strong channels leaves them."""
    x = torch.randn(shape, generator=_gen(seed, stream), device=DEV)
    x.mul_(1 + 3 * (torch.rand(shape[1], generator=_gen(seed, stream + 1), device=DEV) < 0.01))
    return (x * torch.rsqrt(x.pow(2).mean(-1, keepdim=True) + EPS)).to(torch.bfloat16)


def _empty(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device=DEV)


def _copy_buffers(r, c, both):
    s = {"q": _empty(r, c, dtype=torch.uint8), "q_scale": _empty(r // 128, (c // 128 + 3) // 4, 512, dtype=torch.uint8)}
    if both:
        s["q_t"] = _empty(c, r, dtype=torch.uint8)
        s["q_t_scale"] = _empty(c // 128, (r // 128 + 3) // 4, 512, dtype=torch.uint8)
    return s


def prepare(case, seed):
    kind = case["kind"]
    s = {"case": case, "status": torch.zeros(1, dtype=torch.int32, device=DEV)}
    if kind.startswith("qk"):
        t, hq, hkv, d, rot = (case[n] for n in ("t", "hq", "hkv", "d", "rot"))
        qkv = _normal((t, (hq + 2 * hkv) * d), 1.0, seed, 0)
        qkv.mul_(torch.rand(t, 1, generator=_gen(seed, 1), device=DEV).add_(0.5).to(torch.bfloat16))
        s["q"] = qkv[:, :hq * d].view(t, hq, d)
        s["k"] = qkv[:, hq * d:(hq + hkv) * d].view(t, hkv, d)
        s["q_gain"], s["k_gain"] = (_normal((d,), 0.2, seed, 2 + i).add_(1) for i in range(2))
        # positions start again at each packed sequence; the padding rows behind the last one are at -1
        used = t - case["pad"]
        cuts = torch.linspace(0, used, case["seqs"] + 1).round().int().tolist()
        pos = torch.full((t,), -1, dtype=torch.int32)
        for a, b in zip(cuts[:-1], cuts[1:]):
            pos[a:b] = torch.arange(b - a, dtype=torch.int32) + (seed % 1000 if t == 1 else 0)
        s["positions"] = pos.to(DEV)
        ang = torch.arange(int(pos.max()) + 1, dtype=torch.float64, device=DEV)[:, None] * \
            ROPE_BASE ** (-2 * torch.arange(rot // 2, dtype=torch.float64, device=DEV) / rot)
        s["cos"], s["sin"] = ang.cos().float(), ang.sin().float()
        s["rstd"] = _empty(t, hq + hkv, dtype=torch.float32)
        if kind == "qk":
            s["q_out"], s["k_out"] = _empty(t, hq, d), _empty(t, hkv, d)
        else:
            s["dq_out"], s["dk_out"] = _normal((t, hq, d), 1e-3, seed, 4), _normal((t, hkv, d), 1e-3, seed, 5)
            x = torch.cat([s["q"], s["k"]], 1).float()
            s["rstd"] = (1 / torch.sqrt(x.pow(2).mean(-1) + EPS)) * (s["positions"] >= 0)[:, None]
            dqkv = _empty(t, (hq + 2 * hkv) * d)
            s["dq"], s["dk"] = dqkv[:, :hq * d].view(t, hq, d), dqkv[:, hq * d:(hq + hkv) * d].view(t, hkv, d)
            s["dq_gain"], s["dk_gain"] = _empty(d, dtype=torch.float32), _empty(d, dtype=torch.float32)
            s["workspace"] = _empty(4 << 20, dtype=torch.uint8)
    elif kind == "linear":
        m, n, k, ops = (case[i] for i in ("m", "n", "k", "ops"))
        s["x"] = _operand(_normed((m, k), seed, 0), ops, False)
        s["w"] = _operand(_normal((n, k), 0.02, seed, 2), ops, True)
        s["bias"] = _normal((n,), 0.3, seed, 3) if case["bias"] else None
        s["residual"] = _normal((m, n), 1.0, seed, 4) if case["residual"] else None
        s["y"], s["z"] = _empty(m, n), _empty(m, n) if case["z"] else None
        s["workspace"] = _empty(8 * ((m + 255) // 256 * 256) * n * 4, dtype=torch.uint8) if m <= 4096 else None
    elif kind == "act_backward":
        m, n = case["m"], case["n"]
        s["dy"] = _normal((m, n), 1e-3, seed, 0)
        s["z"] = _normal((m, n), 1.0, seed, 1) if case["act"] != "none" else None
        s["dbias"] = _empty(n, dtype=torch.float32) if case["dbias"] else None
        s["workspace"] = _empty(max(1024, (m + 127) // 128 * 4 * n * 4), dtype=torch.uint8)
        s |= _copy_buffers(m, n, True) if case["ops"] == "block" else {"dz": _empty(m, n)}
    elif kind == "gated":
        m, f, k, ops = (case[i] for i in ("m", "f", "k", "ops"))
        s["x"] = _operand(_normed((m, k), seed, 0), ops, False)
        s["w"] = _operand(_normal((2 * f, k), 0.02, seed, 2), ops, True)
        s["gate_up"] = _empty(m, 2 * f) if case["keep"] else None
        s |= _copy_buffers(m, f, True) if ops == "block" else {"h": _empty(m, f)}
    else:
        m, f = case["m"], case["f"]
        gate_up = _normal((m, 2 * f), 1.0, seed, 0)
        s["gate"], s["up"] = gate_up[:, :f], gate_up[:, f:]
        s["dh"] = _normal((m, f), 1e-3, seed, 1)
        s |= _copy_buffers(m, 2 * f, True) if case["ops"] == "block" else {"dgate_up": _empty(m, 2 * f)}
    if own:
        import paper_2608_27370_gb300 as P

        s["P"] = P
        if kind in ("linear", "gated") and case["ops"] != "bf16":
            scaling = P.SCALE_BLOCK if case["ops"] == "block" else P.SCALE_TENSOR
            for n, role in (("x", P.ROLE_ACT), ("w", P.ROLE_WEIGHT)):
                s[n + "_op"] = P.FP8Operand(s[n]["codes"], s[n]["scale"], P.E4M3, scaling, role)
        s["act"] = getattr(P, "ACT_" + case["act"].upper()) if "act" in case else None
        s["fmt"] = getattr(P, case["fmt"].upper()) if "fmt" in case else None
    return s


# ------------------------------------------------------------- the definitions, in the type of their inputs
def _rotate(x, cos, sin, rot, inter, back):
    """R x, or R^T x: pairs (i, i + rot / 2), or neighbours, turned by the position's angles; x [T, H, D]."""
    if back:
        sin = -sin
    c, s = cos[:, None, :], sin[:, None, :]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if inter else (x[..., :rot // 2], x[..., rot // 2:rot])
    p, q = a * c - b * s, b * c + a * s
    turned = torch.stack([p, q], -1).flatten(-2) if inter else torch.cat([p, q], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _qk(s, dtype):
    case, pos = s["case"], s["positions"]
    live = (pos >= 0)[:, None, None]
    at = pos.clamp(min=0).long()
    cos, sin = s["cos"].to(dtype)[at], s["sin"].to(dtype)[at]
    out, rstd = [], []
    for x, gain in ((s["q"], s["q_gain"]), (s["k"], s["k_gain"])):
        x = x.to(dtype)
        r = 1 / torch.sqrt(x.pow(2).mean(-1, keepdim=True) + EPS)
        y = _rotate(x * r * gain.to(dtype), cos, sin, case["rot"], case["inter"], False)
        out.append(torch.where(live, y, torch.zeros_like(y)))
        rstd.append(torch.where(live, r, torch.zeros_like(r))[..., 0])
    return out[0], out[1], torch.cat(rstd, 1)


def _qk_backward(s, dtype):
    case, pos = s["case"], s["positions"]
    live = (pos >= 0)[:, None, None]
    at = pos.clamp(min=0).long()
    cos, sin = s["cos"].to(dtype)[at], s["sin"].to(dtype)[at]
    hq = case["hq"]
    out, gains = [], []
    for dy, x, r, gain in ((s["dq_out"], s["q"], s["rstd"][:, :hq], s["q_gain"]), (s["dk_out"], s["k"], s["rstd"][:, hq:], s["k_gain"])):
        dn = _rotate(dy.to(dtype), cos, sin, case["rot"], case["inter"], True)
        r = r.to(dtype)[..., None]
        xh = x.to(dtype) * r
        dn = torch.where(live, dn, torch.zeros_like(dn))
        gains.append((dn * xh).sum((0, 1)))
        dx = dn * gain.to(dtype)
        out.append(r * (dx - xh * (dx * xh).mean(-1, keepdim=True)))
    return out[0], out[1], gains[0], gains[1]


def _linear(s, dtype):
    case = s["case"]
    z = _values(s["x"], case["ops"], dtype) @ _values(s["w"], case["ops"], dtype).t()
    if s["bias"] is not None:
        z = z + s["bias"].to(dtype)
    y = _act(z, case["act"])
    return (y if s["residual"] is None else y + s["residual"].to(dtype)), z


def _act_backward(s, dtype):
    case = s["case"]
    dz = s["dy"].to(dtype)
    if s["z"] is not None:
        dz = dz * _act_slope(s["z"].to(dtype), case["act"])
    return dz, dz.sum(0)


def _gated(s, dtype):
    case = s["case"]
    gu = _values(s["x"], case["ops"], dtype) @ _values(s["w"], case["ops"], dtype).t()
    return gu, _act(gu[:, :case["f"]], case["act"]) * gu[:, case["f"]:]


def _gated_backward(s, dtype):
    act = s["case"]["act"]
    dh, g, u = s["dh"].to(dtype), s["gate"].to(dtype), s["up"].to(dtype)
    return torch.cat([dh * u * _act_slope(g, act), dh * _act(g, act)], 1)


# ------------------------------------------------------------- one pass
def _run_plain(s):
    case = s["case"]
    kind, bf = case["kind"], torch.bfloat16
    if kind == "qk":
        q, k, rstd = _qk(s, torch.float32)
        return {"q": q.to(bf), "k": k.to(bf), "rstd": rstd}
    if kind == "qk_backward":
        dq, dk, gq, gk = _qk_backward(s, torch.float32)
        return {"dq": dq.to(bf), "dk": dk.to(bf), "dq_gain": gq, "dk_gain": gk}
    if kind == "linear":
        y, z = _linear(s, torch.float32)
        return {"y": y.to(bf), **({"z": z.to(bf)} if case["z"] else {})}
    if kind == "act_backward":
        dz, db = _act_backward(s, torch.float32)
        out = _copies(dz, case["fmt"], True) if case["ops"] == "block" else {"dz": dz.to(bf)}
        return {**out, **({"dbias": db} if case["dbias"] else {})}
    if kind == "gated":
        gu, h = _gated(s, torch.float32)
        out = _copies(h, case["fmt"], True) if case["ops"] == "block" else {"h": h.to(bf)}
        return {**out, **({"gate_up": gu.to(bf)} if case["keep"] else {})}
    d = _gated_backward(s, torch.float32)
    return _copies(d, case["fmt"], True) if case["ops"] == "block" else {"dgate_up": d.to(bf)}


def _run_own(s):
    case, P = s["case"], s["P"]
    kind = case["kind"]
    if kind == "qk":
        P.puro_qk_norm_rope(s["q"], s["k"], s["q_gain"], s["k_gain"], EPS, s["cos"], s["sin"], s["positions"], case["inter"],
                            s["q_out"], s["k_out"], s["rstd"], dev_status=s["status"])
        return {"q": s["q_out"], "k": s["k_out"], "rstd": s["rstd"]}
    if kind == "qk_backward":
        P.puro_qk_norm_rope_backward(s["dq_out"], s["dk_out"], s["q"], s["k"], s["rstd"], s["q_gain"], s["k_gain"], s["cos"],
                                     s["sin"], s["positions"], case["inter"], s["dq"], s["dk"], s["dq_gain"], s["dk_gain"],
                                     s["workspace"], dev_status=s["status"])
        return {n: s[n] for n in ("dq", "dk", "dq_gain", "dk_gain")}
    copies = [s.get(n) for n in ("q", "q_scale", "q_t", "q_t_scale")]
    if kind == "linear":
        if case["ops"] == "bf16":
            P.puro_bf16_linear_fprop_epilogue(s["x"]["x"], s["w"]["x"], s["y"], s["bias"], s["act"], s["residual"], s["z"],
                                              dev_status=s["status"])
        else:
            P.puro_fp8_linear_fprop_epilogue(s["x_op"], s["w_op"], s["y"], s["bias"], s["act"], s["residual"], s["z"],
                                             s["workspace"], dev_status=s["status"])
        return {"y": s["y"], **({"z": s["z"]} if case["z"] else {})}
    if kind == "act_backward":
        if case["ops"] == "block":
            P.puro_fp8_quantize_act_backward(s["dy"], s["z"], s["act"], s["fmt"], None, s["dbias"], s["workspace"], *copies,
                                             dev_status=s["status"])
        else:
            P.puro_act_backward_bf16(s["dy"], s["z"], s["act"], s["dz"], s["dbias"], s["workspace"])
        out = _own_copies(s) if case["ops"] == "block" else {"dz": s["dz"]}
        return {**out, **({"dbias": s["dbias"]} if case["dbias"] else {})}
    if kind == "gated":
        if case["ops"] == "block":
            P.puro_fp8_gated_fprop(s["x_op"], s["w_op"], s["act"], s["fmt"], s["gate_up"], None, *copies, dev_status=s["status"])
        else:
            P.puro_bf16_gated_fprop(s["x"]["x"], s["w"]["x"], s["act"], s["gate_up"], s["h"], dev_status=s["status"])
        out = _own_copies(s) if case["ops"] == "block" else {"h": s["h"]}
        return {**out, **({"gate_up": s["gate_up"]} if case["keep"] else {})}
    if case["ops"] == "block":
        P.puro_fp8_quantize_gated_backward(s["dh"], s["gate"], s["up"], s["act"], s["fmt"], None, *copies, dev_status=s["status"])
        return _own_copies(s)
    P.puro_gated_backward_bf16(s["dh"], s["gate"], s["up"], s["act"], s["dgate_up"])
    return {"dgate_up": s["dgate_up"]}


def _own_copies(s):
    f8 = F8[s["case"]["fmt"]]
    return {"q": s["q"].view(f8), "q_scale": s["q_scale"].view(torch.float8_e8m0fnu), "q_t": s["q_t"].view(f8),
            "q_t_scale": s["q_t_scale"].view(torch.float8_e8m0fnu)}


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    kind = case["kind"]
    if kind.startswith("qk"):
        live, heads = case["t"] - case["pad"], case["hq"] + case["hkv"]
        row = heads * case["d"] * 2
        longest = -(-live // case["seqs"])  # rows of the tables that the positions reach
        other = 4 * case["t"] + 4 * case["t"] * heads + 4 * longest * case["rot"] + 4 * case["d"]
        back = kind == "qk_backward"
        return {"bytes": (2 if back else 1) * live * row + case["t"] * row + other + (8 * case["d"] if back else 0),
                "flops": (14 if back else 8) * live * heads * case["d"]}
    copies = 2 * (1 + 1 / 128)  # the two FP8 copies of a value with their scales
    block = case.get("ops") == "block"
    m, n = case["m"], case.get("n", case.get("f"))
    eb = 2 if case.get("ops") == "bf16" else 1 + (1 / 128 if block else 0)
    if kind == "linear":
        k = case["k"]
        return {"bytes": eb * (m + n) * k + 2 * n * case["bias"] + 2 * m * n * (1 + case["residual"] + case["z"]), "flops": 2 * m * n * k}
    if kind == "act_backward":
        return {"bytes": m * n * ((4 if case["act"] != "none" else 2) + (copies if block else 2)) + 4 * n * case["dbias"],
                "flops": 10 * m * n}
    if kind == "gated":
        k = case["k"]
        return {"bytes": eb * (m + 2 * n) * k + m * n * ((copies if block else 2) + 4 * case["keep"]), "flops": 4 * m * n * k}
    return {"bytes": m * n * (6 + 2 * (copies if block else 2)), "flops": 16 * m * n}


def exact(case, seed):
    """The definitions in 64 bits on the same inputs; a copy's numbers before their rounding to 8 bits."""
    s = prepare(case, seed)
    kind, d = case["kind"], torch.float64
    if kind == "qk":
        return dict(zip(("q", "k", "rstd"), _exact_qk(s)))
    if kind == "qk_backward":
        return dict(zip(("dq", "dk", "dq_gain", "dk_gain"), _exact_qk_backward(s)))
    if kind == "linear":
        x, w = _values(s["x"], case["ops"], d), _values(s["w"], case["ops"], d)
        z = torch.einsum("mk,nk->mn", x, w)
        if case["bias"]:
            z += s["bias"].double()
        y = _exact_act(z, case["act"])[0]
        return {"y": y + s["residual"].double() if case["residual"] else y, **({"z": z} if case["z"] else {})}
    if kind == "act_backward":
        dz = s["dy"].double()
        if case["act"] != "none":
            dz = dz * _exact_act(s["z"].double(), case["act"])[1]
        out = _exact_copies(dz, case["fmt"], True) if case["ops"] == "block" else {"dz": dz}
        return {**out, **({"dbias": dz.sum(0)} if case["dbias"] else {})}
    if kind == "gated":
        f = case["f"]
        x, w = _values(s["x"], case["ops"], d), _values(s["w"], case["ops"], d)
        gate, up = torch.einsum("mk,nk->mn", x, w[:f]), torch.einsum("mk,nk->mn", x, w[f:])
        h = _exact_act(gate, case["act"])[0] * up
        out = _exact_copies(h, case["fmt"], True) if case["ops"] == "block" else {"h": h}
        return {**out, **({"gate_up": torch.cat([gate, up], 1)} if case["keep"] else {})}
    a, slope = _exact_act(s["gate"].double(), case["act"])
    dgu = torch.empty(case["m"], 2 * case["f"], dtype=d, device=DEV)
    dgu[:, :case["f"]] = s["dh"].double() * s["up"].double() * slope
    dgu[:, case["f"]:] = s["dh"].double() * a
    return _exact_copies(dgu, case["fmt"], True) if case["ops"] == "block" else {"dgate_up": dgu}


def _exact_act(z, act):
    """The activation and its slope, from tanh and erf, apart from the plain form."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return z.clamp(min=0), (z > 0).double()
    if act == "silu":
        t = torch.tanh(z / 2)
        return z * (1 + t) / 2, (1 + t) / 2 + z * (1 - t * t) / 4
    if act == "gelu":
        p = (1 + torch.erf(z / math.sqrt(2))) / 2
        return z * p, p + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    a = math.sqrt(2 / math.pi)
    t = torch.tanh(a * (z + 0.044715 * z * z * z))
    return z * (1 + t) / 2, (1 + t) / 2 + z * (1 - t * t) / 2 * a * (1 + 0.134145 * z * z)


def _exact_turn(s, sign):
    """e^{sign i angle} for each token and pair, as complex numbers."""
    at = s["positions"].clamp(min=0).long()
    return torch.complex(s["cos"].double()[at], sign * s["sin"].double()[at])[:, None, :]


def _exact_turned(x, turn, case):
    rot = case["rot"]
    y = x.clone()
    if case["inter"]:
        z = torch.complex(x[..., 0:rot:2], x[..., 1:rot:2]) * turn
        y[..., 0:rot:2], y[..., 1:rot:2] = z.real, z.imag
    else:
        z = torch.complex(x[..., :rot // 2], x[..., rot // 2:rot]) * turn
        y[..., :rot // 2], y[..., rot // 2:rot] = z.real, z.imag
    return y


def _exact_qk(s):
    case, live = s["case"], (s["positions"] >= 0).double()[:, None, None]
    turn = _exact_turn(s, 1.0)
    out, rs = [], []
    for x, g in ((s["q"].double(), s["q_gain"].double()), (s["k"].double(), s["k_gain"].double())):
        r = (torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / case["d"] + EPS) ** -0.5
        out.append(_exact_turned(x * r * g, turn, case) * live)
        rs.append((r * live)[..., 0])
    return out[0], out[1], torch.cat(rs, 1)


def _exact_qk_backward(s):
    case, live = s["case"], (s["positions"] >= 0).double()[:, None, None]
    turn, hq, d = _exact_turn(s, -1.0), s["case"]["hq"], s["case"]["d"]
    res = []
    for dy, x, r, g in ((s["dq_out"], s["q"], s["rstd"][:, :hq], s["q_gain"]), (s["dk_out"], s["k"], s["rstd"][:, hq:], s["k_gain"])):
        dn = _exact_turned(dy.double(), turn, case) * live
        x, r, g = x.double(), r.double()[..., None], g.double()
        # dx = r g dn - x r^3 (sum g dn x) / d
        dx = r * g * dn - x * r ** 3 * torch.einsum("thd,thd,d->th", dn, x, g)[..., None] / d
        res.append((dx, torch.einsum("thd,thd,th->d", dn, x, r[..., 0])))
    return res[0][0], res[1][0], res[0][1], res[1][1]
