"""The operators that the training step of a decoder layer needs around its
linears and the MuonH step, each through one public call: what is measured,
their plain form and their exact results.

Kinds of case
  muon           the Muon directions of some matrices, in one call: momentum, then
                 X = V / |V|_F and steps X <- a X + (b A + c A^2) X, A = X X^T
  rope           the position rotation of queries and keys without a norm, angles
                 from the positions, frequencies scaled for long contexts
  rope_backward  its gradient: the transposed rotation of dq and dk
  rope_tables    cosines and sines of positions in FP32, as the norms with a rotation
                 read them

A muon case's "shapes" is "COUNTxROWSxCOLS,...": that many matrices of one shape,
whose gradients, momenta and directions a program keeps in one tensor each.
"""
import math

import torch

own = False

DEV = "cuda"
STEPS = ((3.4445, -4.7750, 2.0315),) * 5
MU = 0.95
MAX_FLOPS = 3.2e12  # of the largest listed case's directions, about


def listed():
    return [
        # one Qwen2-1.5B layer's matrices as the optimiser of a data-parallel trainer gets them: FP32 main gradients
        dict(name="muon_layer", kind="muon", shapes="1x2048x1536,1x1536x1536,2x8960x1536,1x1536x8960", grad="fp32",
             momentum=True, nesterov=True, pad=0),
        # two Qwen3-1.7B layers together, BF16 gradients
        dict(name="muon_two_layers", kind="muon", shapes="2x4096x2048,2x2048x2048,4x6144x2048,2x2048x6144", grad="bf16",
             momentum=True, nesterov=True, pad=0),
        # one square matrix alone, as a sharded optimiser hands them out; no momentum
        dict(name="muon_one", kind="muon", shapes="1x1536x1536", grad="bf16", momentum=False, nesterov=False, pad=0),
        # many small matrices of odd sizes (projections of single heads, adapters)
        dict(name="muon_heads", kind="muon", shapes="24x128x1536,3x257x129,8x1536x64", grad="bf16", momentum=True, nesterov=False, pad=3),
        # a tiny one: nothing but latency
        dict(name="muon_tiny", kind="muon", shapes="1x48x80", grad="fp32", momentum=True, nesterov=True, pad=0),
        # the Qwen2-1.5B queries and keys of the benchmark's step
        dict(name="rope_m32768", kind="rope", t=32768, hq=12, hkv=2, d=128, rot=128, inter=False, seqs=8, pad=0, scaling="none",
             factor=1.0, first=0),
        # one token far into a context stretched eightfold
        dict(name="rope_token", kind="rope", t=1, hq=12, hkv=2, d=128, rot=128, inter=False, seqs=1, pad=0, scaling="index",
             factor=8.0, first=131071),
        # the gradient at the paper's micro-batch
        dict(name="rope_backward_m8192", kind="rope_backward", t=8192, hq=16, hkv=8, d=128, rot=128, inter=False, seqs=2, pad=0,
             scaling="none", factor=1.0, first=0),
        # packed sequences of odd lengths with padding rows behind them, half of each head in neighbouring pairs, stretched
        dict(name="rope_backward_ragged", kind="rope_backward", t=5003, hq=12, hkv=2, d=128, rot=64, inter=True, seqs=7, pad=37,
             scaling="turns", factor=4.0, first=0),
        # the tables of a long context
        dict(name="rope_tables_131072", kind="rope_tables", t=131072, rot=128, scaling="index", factor=4.0, first=0),
        # some rows of them, far out
        dict(name="rope_tables_rows", kind="rope_tables", t=37, rot=64, scaling="base", factor=8.0, first=1000003),
    ]


def _log(rng, lo, hi, step=1):
    """A multiple of step between lo and hi, even over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step))


def _scaling(rng):
    kind = rng.choice(["none", "linear", "base", "turns", "index"])
    return dict(scaling=kind, factor=1.0 if kind == "none" else rng.choice([2.0, 4.0, 5.5, 8.0, 32.0]))


def draw(rng):
    kind = rng.choice(["muon", "muon", "rope", "rope_backward", "rope_tables"])
    if kind == "muon":
        shapes, left = [], MAX_FLOPS / 2
        for _ in range(rng.randint(1, 3)):
            r, c = _log(rng, 4, 6144), _log(rng, 4, 6144)
            r, c = min(r, 4 * c, 9216), min(c, 9216)
            if rng.random() < 0.5:
                r, c = (r + 7) // 8 * 8, (c + 7) // 8 * 8
            one = _muon_flops(r, c)
            if one > left:
                continue
            n = max(1, min(rng.randint(1, 12), int(left / one)))
            left -= n * one
            shapes.append("%dx%dx%d" % (n, r, c))
        return dict(kind=kind, shapes=",".join(shapes or ["2x%dx%d" % (rng.randint(9, 900), rng.randint(9, 900))]),
                    grad=rng.choice(["fp32", "bf16"]), momentum=rng.random() < 0.7, nesterov=rng.random() < 0.5,
                    pad=rng.choice([0, 0, 1, 8]))
    if kind == "rope_tables":
        return dict(kind=kind, t=_log(rng, 1, 131072), rot=rng.choice([32, 64, 96, 128, 256]), first=rng.choice([0, _log(rng, 1, 4000000)]),
                    **_scaling(rng))
    d = rng.choice([64, 80, 96, 128, 192, 256])
    t = _log(rng, 1, 16384)
    hkv = rng.choice([1, 2, 4, 8])
    return dict(kind=kind, t=t, hq=hkv * rng.choice([1, 2, 4, 6]) if d <= 128 else hkv, hkv=hkv, d=d,
                rot=rng.choice([d, d // 2 // 16 * 16]), inter=rng.random() < 0.3, seqs=rng.randint(1, max(1, min(8, t))),
                pad=rng.choice([0, 0, t // 9]), first=rng.choice([0, _log(rng, 1, 1000000)]), **_scaling(rng))


def _shapes(case):
    return [tuple(int(v) for v in s.split("x")) for s in case["shapes"].split(",")]


def _muon_flops(r, c):
    """Of one matrix's direction, a symmetric product counted once."""
    m, n = min(r, c), max(r, c)
    return len(STEPS) * (3 * m * m * n + m ** 3)


def work(case):
    kind = case["kind"]
    if kind == "muon":
        values = sum(n * r * c for n, r, c in _shapes(case))
        per = (4 if case["grad"] == "fp32" else 2) + (8 if case["momentum"] else 0) + 2
        return {"bytes": per * values, "flops": sum(n * _muon_flops(r, c) for n, r, c in _shapes(case))}
    if kind == "rope_tables":
        return {"bytes": 4 * case["t"] * case["rot"], "flops": 4 * case["t"] * case["rot"]}
    values = case["t"] * (case["hq"] + case["hkv"]) * case["d"]
    return {"bytes": 4 * values + 4 * case["t"], "flops": 3 * values}


# ------------------------------------------------------------- inputs
def _gen(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed(64 * seed + stream)
    return g


def _normal(shape, std, seed, stream):
    return torch.randn(shape, generator=_gen(seed, stream), device=DEV).mul_(std)


def _gradients(n, r, c, seed, stream):
    """A few strong directions, as batches agree on them, and noise in all: [n, r, c] in FP32."""
    k = max(1, min(r, c, 16) // 2)
    strong = _normal((n, r, k), 1.0, seed, stream) @ _normal((n, k, c), 1.0 / math.sqrt(k), seed, stream + 1)
    rows = torch.rand((n, r, 1), generator=_gen(seed, stream + 2), device=DEV).add_(0.5)
    return (strong + _normal((n, r, c), 0.5, seed, stream + 3)).mul_(rows).mul_(1e-4)


def _frequencies(case):
    """The angle of each pair per position, scaled for a context factor times the trained one of 32768: fp64 [rot / 2]."""
    base, trained, rot, f = 1e6, 32768.0, case["rot"], case["factor"]
    i = torch.arange(rot // 2, dtype=torch.float64)
    if case["scaling"] == "base":
        base = base * f ** (rot / (rot - 2))
    w = base ** (-2 * i / rot)
    if case["scaling"] == "linear":
        w = w / f
    elif case["scaling"] == "turns":  # pairs of few turns over the trained context are slowed down, of many kept
        keep = ((trained * w / (2 * math.pi) - 1) / (32 - 1)).clamp(0, 1)
        w = (1 - keep) * w / f + keep * w
    elif case["scaling"] == "index":  # the same between the pairs of 32 turns and of one, even over their indexes
        lo, hi = (rot * math.log(trained / (turns * 2 * math.pi)) / (2 * math.log(base)) for turns in (32.0, 1.0))
        lo, hi = max(0, math.floor(lo)), min(rot // 2 - 1, math.ceil(hi))
        keep = 1 - ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        w = (1 - keep) * w / f + keep * w
    return w.to(DEV)


def _attention_scale(case):
    return 0.1 * math.log(case["factor"]) + 1 if case["scaling"] in ("turns", "index") else 1.0


def prepare(case, seed):
    s = {"case": case}
    kind = case["kind"]
    if kind == "muon":
        s["grads"], s["momenta"], s["u"] = [], [], []
        for j, (n, r, c) in enumerate(_shapes(case)):
            g = torch.zeros((n, r, c + case["pad"]), dtype=torch.float32 if case["grad"] == "fp32" else torch.bfloat16, device=DEV)
            g[..., :c] = _gradients(n, r, c, seed, 8 * j)
            s["grads"].append(g[..., :c])
            s["momenta"].append(_gradients(n, r, c, seed, 8 * j + 4).mul_(4.0) if case["momentum"] else None)
            s["u"].append(torch.empty((n, r, c), dtype=torch.bfloat16, device=DEV))
    else:
        s["w"], s["scale"] = _frequencies(case), _attention_scale(case)
    if kind == "rope_tables":
        s["first"] = case["first"] + seed % 1000  # another seed: other positions
        s["cos"], s["sin"] = (torch.empty((case["t"], case["rot"] // 2), device=DEV) for _ in range(2))
    elif kind != "muon":
        t, hq, hkv, d = (case[n] for n in ("t", "hq", "hkv", "d"))
        # positions start again at each packed sequence; the padding rows behind the last one are at -1
        used = t - case["pad"]
        cuts = torch.linspace(0, used, case["seqs"] + 1).round().int().tolist()
        pos = torch.full((t,), -1, dtype=torch.int32)
        for a, b in zip(cuts[:-1], cuts[1:]):
            pos[a:b] = torch.arange(b - a, dtype=torch.int32) + case["first"]
        s["positions"] = pos.to(DEV)
        qkv = _normal((t, (hq + 2 * hkv) * d), 1.0, seed, 0).to(torch.bfloat16)
        qkv.mul_(torch.rand(t, 1, generator=_gen(seed, 1), device=DEV).add_(0.5).to(torch.bfloat16))
        views = (qkv[:, :hq * d].view(t, hq, d), qkv[:, hq * d:(hq + hkv) * d].view(t, hkv, d))
        whole = tuple(torch.empty((t, h, d), dtype=torch.bfloat16, device=DEV) for h in (hq, hkv))
        if kind == "rope":
            s["x"], s["y"] = views, whole
        else:  # dq and dk whole, into their places in the gradient of the qkv output
            s["x"] = tuple(w.copy_(v) for w, v in zip(whole, views))
            s["y"] = tuple(torch.empty_like(qkv)[:, a * d:(a + h) * d].view(t, h, d) for a, h in ((0, hq), (hq, hkv)))
    if own:
        import paper_2608_27370_gb300 as P

        s["P"] = P
        if kind == "muon":
            s["table"] = P.muon_table([(g[i], m[i] if m is not None else None, u[i])
                                       for g, m, u in zip(s["grads"], s["momenta"], s["u"]) for i in range(len(g))])
            s["workspace"] = torch.empty(P.puro_muon_direction_workspace_size(s["table"]), dtype=torch.uint8, device=DEV)
        else:
            s["frequencies"] = P.rope_frequencies(case["rot"], 1e6, getattr(P, "ROPE_" + case["scaling"].upper()), case["factor"], 32768,
                                                  32.0, 1.0, device=DEV)
    return s


# ------------------------------------------------------------- the plain form, in 32 bits (angles in 64)
def _direction(s, k):
    g, m = s["grads"][k].float(), s["momenta"][k]
    if m is not None:
        m.mul_(MU).add_(g)
        g = g + MU * m if s["case"]["nesterov"] else m
    r, c = g.shape[1:]
    x = g / g.double().square().sum((1, 2), keepdim=True).sqrt().float()
    x = x.mT if r > c else x
    for a, b, c2 in STEPS:
        gram = x @ x.mT
        x = a * x + (b * gram + c2 * (gram @ gram)) @ x
    s["u"][k].copy_(x.mT if r > c else x)


def _cos_sin(s, pos):
    angle = pos.double()[:, None] * s["w"]
    return (s["scale"] * angle.cos()).float(), (s["scale"] * angle.sin()).float()


def _turned(s, x, cos, sin):
    rot, live = s["case"]["rot"], (s["positions"] >= 0)[:, None, None]
    x = x.float()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if s["case"]["inter"] else (x[..., :rot // 2], x[..., rot // 2:rot])
    p, q = a * cos - b * sin, b * cos + a * sin
    y = torch.stack([p, q], -1).flatten(-2) if s["case"]["inter"] else torch.cat([p, q], -1)
    return torch.where(live, torch.cat([y, x[..., rot:]], -1), torch.zeros_like(x))


def run(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "muon":
        if own:
            s["P"].puro_muon_direction_grouped(s["table"], s["workspace"], MU, case["nesterov"], STEPS)
        else:
            for k in range(len(s["grads"])):
                _direction(s, k)
        return {"u": s["u"], "momenta": s["momenta"]}
    if kind == "rope_tables":
        if own:
            s["P"].puro_rope_tables(s["frequencies"], s["first"], s["cos"], s["sin"], scale=s["scale"])
        else:
            c, n = _cos_sin(s, s["first"] + torch.arange(case["t"], device=DEV))
            s["cos"].copy_(c)
            s["sin"].copy_(n)
        return {"cos": s["cos"], "sin": s["sin"]}
    (q, k), (q_out, k_out) = s["x"], s["y"]
    if own:
        call = s["P"].puro_rope if kind == "rope" else s["P"].puro_rope_backward
        call(q, k, s["frequencies"], s["positions"], case["inter"], q_out, k_out, scale=s["scale"])
    else:
        c, n = (v[:, None, :] for v in _cos_sin(s, s["positions"].clamp(min=0)))
        q_out.copy_(_turned(s, q, c, n if kind == "rope" else -n))
        k_out.copy_(_turned(s, k, c, n if kind == "rope" else -n))
    return {"q": q_out, "k": k_out}


# ------------------------------------------------------------- the definitions in 64 bits, by another road
def _exact_direction(v):
    """P(A0) X0, with A <- A q(A)^2 and P <- q(A) P, q(A) = a + b A + c A^2: the Gram matrices follow from the first."""
    x = v / torch.linalg.matrix_norm(v)
    tall = x.shape[0] > x.shape[1]
    gram = x.T @ x if tall else x @ x.T
    eye = torch.eye(len(gram), dtype=torch.float64, device=v.device)
    p = eye
    for a, b, c in STEPS:
        q = torch.addmm(a * eye, gram, b * eye + c * gram)
        p = q @ p
        gram = q @ gram @ q
    return x @ p if tall else p @ x


def exact(case, seed):
    if case["kind"] == "muon" and work(case)["flops"] > 8e12:
        return None
    s = prepare(case, seed)
    if case["kind"] == "muon":
        momenta, u = [], []
        for g, m in zip(s["grads"], s["momenta"]):
            v = g.double()
            if m is not None:
                momenta.append(MU * m.double() + v)
                v = v + MU * momenta[-1] if case["nesterov"] else momenta[-1]
            else:
                momenta.append(None)
            u.append(torch.stack([_exact_direction(x) for x in v]))
        return {"u": u, "momenta": momenta}
    pos = torch.arange(case["t"], device=DEV) + s["first"] if case["kind"] == "rope_tables" else s["positions"].clamp(min=0).long()
    # whole turns of 4096 positions and the rest apart, as complex numbers
    unit = torch.polar(torch.full_like(s["w"], s["scale"]), torch.zeros_like(s["w"]))
    turns = unit * torch.exp(1j * (pos // 4096 * 4096)[:, None] * s["w"]) * torch.exp(1j * (pos % 4096)[:, None] * s["w"])
    if case["kind"] == "rope_tables":
        return {"cos": turns.real.contiguous(), "sin": turns.imag.contiguous()}
    turns = (turns if case["kind"] == "rope" else turns.conj())[:, None, :]
    out = {}
    for name, x in zip("qk", s["x"]):
        y, rot = x.double(), case["rot"]
        at = (slice(0, rot, 2), slice(1, rot, 2)) if case["inter"] else (slice(0, rot // 2), slice(rot // 2, rot))
        z = torch.complex(y[..., at[0]], y[..., at[1]]) * turns
        y[..., at[0]], y[..., at[1]] = z.real, z.imag
        y[s["positions"] < 0] = 0
        out[name] = y
    return out
