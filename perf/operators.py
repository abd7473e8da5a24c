"""Timed cases of the training step's operators around the boundary: what a training program has the
library do between two boundary calls and after the last one.

Every case is a dict with an "op":

  norm     resbm_add_rmsnorm_fwd: the residual's addition and the RMSNorm of the sum, H = X + A and
           N = RMSNorm(H) * gamma, in the activations' type ("out" holds n), in e4m3 with fp32 scales (q),
           or both
  train    the same forward, then its backward (resbm_rmsnorm_bwd): dX = dA = dH + dN . dN/dH, dgamma
  adamw    resbm_adamw_step over the tensors of a model: 32-bit or 8-bit states, fp32 or bf16 weights and
           gradients, bf16 weights with or without an fp32 master copy; with "clip", resbm_grad_norm first
           and the step reads its coefficient
  gnorm    resbm_grad_norm: the global norm of a model's gradients and the clipping coefficient

The plain forms here are elementary torch operations in fp32 (the library's own calls run where `own` is
true). The tensors of a model lie in one buffer per kind, each from a multiple of 256 elements on, with
zeros between them, so that the plain forms take all tensors at once.
"""
import math
import random

import torch

own = False

EPS = 1e-5
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
E4M3 = torch.float8_e4m3fn
E4M3_MAX = 448.0
E4M3_LEAST = 2.0 ** -9       # the smallest e4m3 value above zero
SCALE_LEAST = 2.0 ** -100    # a group's largest magnitude counts as no less than this
BLOCK = 256                  # elements behind one scale of an 8-bit state
HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01)
MAX_NORM = 1.0
MOST_ELEMS = 65536 * 4096    # activations: the headline workload's T x d
MOST_PARAMS = 200_000_000    # drawn models: under the listed stage's


def _norm(name, T, d, op="norm", **kw):
    case = {"name": name, "op": op, "T": T, "d": d, "dtype": "bf16", "residual": True, "out": "n", "group": 0, "pad": 0}
    case.update(kw)
    return case


def _model(name, op, **kw):
    case = {"name": name, "op": op, "layers": 0, "d": 2048, "ffn": 5632, "r": 16, "m": 16, "count": 0, "most": 0,
            "sizes": 0, "w": "bf16", "g": "bf16", "master": False, "bits": 32, "clip": False, "offset": 0}
    case.update(kw)
    return case


def listed():
    return [
        # One token's norm before a projection in 8 bits, one scale a row: the smallest call, latency.
        _norm("norm_token_q8", 1, 4096, out="q"),
        # The second norm of every block of the simulated pipeline (batch 8 x seq 2048).
        _norm("norm_pipeline", 16384, 2048),
        # The headline workload's width, 8-bit output with a scale per 128 columns, the residual stream kept.
        _norm("norm_large_q8", 65536, 4096, out="q", group=128),
        # An odd width in rows that are a slice of a wider buffer, fp32.
        _norm("norm_ragged_f32", 5001, 1003, dtype="f32", pad=21),
        # A block's norm in training, forward and backward.
        _norm("train_pipeline", 16384, 2048, op="train"),
        # A short odd microbatch, forward and backward.
        _norm("train_ragged", 333, 1000, op="train"),
        # The boundaries' own weights (d = 2048, r = m = 16), whose gradients the library gives in fp32.
        _model("adamw_boundary", "adamw", g="f32"),
        # One of the pipeline's four stages (6 layers, SwiGLU 5632 and its boundaries), clipped.
        _model("adamw_stage", "adamw", layers=6, clip=True),
        # The same stage with 8-bit states.
        _model("adamw_stage_8bit", "adamw", layers=6, bits=8),
        # Many ragged tensors, fp32 master copies of bf16 weights, none aligned to more than one element.
        _model("adamw_ragged_8bit", "adamw", count=150, most=400_000, sizes=3, g="f32", master=True, bits=8, offset=1),
        # The gradients of the convergence comparison's model (4 layers, d = 512, SwiGLU 1024).
        _model("gnorm_convergence", "gnorm", layers=4, d=512, ffn=1024),
        # The gradients of a stage.
        _model("gnorm_stage", "gnorm", layers=6),
    ]


def draw(rng):
    log = lambda a, b: int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))
    op = rng.choice(("norm", "norm", "train", "adamw", "adamw", "adamw", "gnorm"))
    if op in ("norm", "train"):
        d = log(64, 8192)
        if rng.random() < 0.6:
            d = max(8, d // 8 * 8)
        T = log(1, min(65536, MOST_ELEMS // d))
        case = {"op": op, "T": T, "d": d, "dtype": rng.choice(("bf16", "bf16", "f32")), "residual": op == "train" or rng.random() < 0.7,
                "out": "n", "group": 0, "pad": 0}
        if op == "norm":
            case["out"] = rng.choice(("n", "q", "nq"))
            case["group"] = rng.choice((0, 32, 64, 128, 256)) if "q" in case["out"] else 0
            case["pad"] = rng.choice((0, 0, 8, 24, 5))
        return case
    case = _model(None, op, r=rng.choice((16, 32)), m=rng.choice((16, 32)), w=rng.choice(("bf16", "bf16", "f32")))
    del case["name"]
    case["g"] = "f32" if case["w"] == "f32" else rng.choice(("bf16", "f32"))
    if rng.random() < 0.5:
        case["d"] = log(128, 4096) // 8 * 8
        case["ffn"] = case["d"] * rng.choice((2, 3)) + 8 * rng.randrange(9)
        each = 4 * case["d"] ** 2 + 3 * case["d"] * case["ffn"]
        case["layers"] = min(rng.randrange(0, 9), MOST_PARAMS // each)
    else:
        case["count"], case["most"], case["sizes"] = log(1, 500), log(3, 400_000), rng.randrange(1 << 20)
    if op == "adamw":
        case["master"] = case["w"] == "bf16" and rng.random() < 0.3
        case["bits"] = rng.choice((32, 8))
        # (a coefficient under one is left to the 32-bit states: next to a rounding border of e4m3 its last bit
        # decides between two codes)
        case["clip"] = case["bits"] == 32 and rng.random() < 0.4
    case["offset"] = rng.choice((0, 0, 0, 1))
    return case


# ---- a model's tensors -------------------------------------------------------------------------
def _sizes(case):
    """Element counts of the model's tensors: the layers of a pipeline stage and its two boundaries' weights, or
    `count` ragged ones."""
    if case["count"]:
        rng = random.Random(case["sizes"])
        return [rng.randint(1, case["most"]) for _ in range(case["count"])]
    d, f, r, m = case["d"], case["ffn"], case["r"], case["m"]
    return [d, d, 3 * d * d, d * d, f * d, f * d, d * f] * case["layers"] + [d * m, m * r, r * m, m * d]


def _slots(case):
    """(start, elements) of every tensor in the buffers, and the buffers' length."""
    at, slots = 0, []
    for n in _sizes(case):
        slots.append((at, n))
        at += -(-n // BLOCK) * BLOCK
    return slots, at


def _flat(total, offset, dtype):
    return torch.zeros(offset + total, dtype=dtype, device="cuda")[offset:]


def _code(x):
    """A buffer in blocks as values in units of the blocks' scales, before their rounding to e4m3, and the scales."""
    b = x.view(-1, BLOCK)
    most = b.abs().amax(dim=1).clamp_min(SCALE_LEAST)
    return (b * (E4M3_MAX / most)[:, None]).clamp(-E4M3_MAX, E4M3_MAX).view(-1), most / E4M3_MAX


def _prepare_model(case, gen):
    slots, total = _slots(case)
    off = case["offset"]
    normal = lambda: torch.randn(total, generator=gen, device="cuda")
    inside = torch.zeros(total, dtype=torch.bool, device="cuda")
    for at, n in slots:
        inside[at:at + n] = True
    # gradients of a model late in training: most of a tensor small, some rows large
    spread = torch.exp(0.7 * torch.randn(total // BLOCK, generator=gen, device="cuda")).repeat_interleave(BLOCK)
    G = _flat(total, off, DT[case["g"]])
    G.copy_(torch.where(inside, normal() * spread * 3e-4, 0.0))
    s = {"slots": slots, "G": G, "step": 1000}
    if case["op"] == "adamw":
        w = torch.where(inside, 0.02 * normal(), 0.0)
        m = torch.where(inside, normal() * spread * 1e-4, 0.0)
        v = torch.where(inside, (normal().abs() + 0.2).square() * spread.square() * 9e-8, 0.0)
        s["W"] = _flat(total, off, DT[case["w"]])
        s["W"].copy_(w)
        if case["master"]:
            s["master"] = _flat(total, off, torch.float32)
            s["master"].copy_(w)
            s["W"].copy_(w)
        if case["bits"] == 8:
            for k, x in (("M", m), ("V", v.sqrt())):
                x, s[k + "s"] = _code(x)
                s[k] = _flat(total, off, E4M3)
                s[k].copy_(x.to(E4M3))
        else:
            for k, x in (("M", m), ("V", v)):
                s[k] = _flat(total, off, torch.float32)
                s[k].copy_(x)
    return s


def _parts(s, key, per=1):
    """The tensors of a model as views of their buffer (per: elements of the model behind one of the buffer's)."""
    if key not in s:
        return None
    return [s[key][at // per:at // per + -(-n // per)] for at, n in s["slots"]]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    if case["op"] in ("adamw", "gnorm"):
        s = _prepare_model(case, gen)
        if own:
            from paper_2604_11947_gb300 import resbm
            if case["op"] == "adamw":
                s["plan"] = resbm.AdamWPlan(_parts(s, "W"), _parts(s, "G"), _parts(s, "M"), _parts(s, "V"),
                                            m_scale=_parts(s, "Ms", BLOCK), v_scale=_parts(s, "Vs", BLOCK),
                                            master=_parts(s, "master"))
            else:
                s["plan"] = resbm.AdamWPlan(None, _parts(s, "G"))
            if case["op"] == "gnorm" or case["clip"]:
                s["out"] = torch.empty(2, device="cuda")
                s["ws"] = resbm.grad_norm_workspace(s["plan"])
        s["case"] = case
        return s
    T, d, dt = case["T"], case["d"], DT[case["dtype"]]

    def rows(scale):
        # activations: N(0, 1) with a log-normal scale per token
        x = torch.randn(T, d + case["pad"], generator=gen, device="cuda")
        x *= scale * torch.exp(0.5 * torch.randn(T, 1, generator=gen, device="cuda"))
        return x.to(dt)[:, :d]

    s = {"case": case, "X": rows(1.0), "A": rows(0.5) if case["residual"] else None,
         "gamma": (1 + 0.1 * torch.randn(d, generator=gen, device="cuda")).to(dt)}
    new = lambda *shape, dtype=dt: torch.empty(*shape, dtype=dtype, device="cuda")
    s["H"] = new(T, d) if case["residual"] else None
    s["N"] = new(T, d) if "n" in case["out"] else None
    s["Q"] = s["S"] = None
    if "q" in case["out"]:
        s["Q"], s["S"] = new(T, d, dtype=E4M3), new(T, -(-d // (case["group"] or d)), dtype=torch.float32)
    if case["op"] == "train":
        s["dN"], s["dH"], s["dX"] = rows(1.0), rows(0.3), new(T, d)
        s["dgamma"] = new(d, dtype=torch.float32)
        if own:
            from paper_2604_11947_gb300 import resbm
            s["desc"] = resbm.make_desc(T, d, 1, 1, case["dtype"])
            s["ws"] = resbm.workspace(s["desc"], resbm.RESBM_OP_RMSNORM_BWD)
    return s


# ---- one pass ----------------------------------------------------------------------------------
def _groups(x, g):
    T, d = x.shape
    return torch.nn.functional.pad(x, (0, -d % g)).view(T, -1, g)


def _plain_norm(s):
    case, gamma = s["case"], s["gamma"].float()
    h = s["X"].float()
    if s["A"] is not None:
        h = h + s["A"].float()
    H = h.to(s["X"].dtype)
    h = H.float()
    rstd = torch.rsqrt(h.square().mean(dim=1, keepdim=True) + EPS)
    n = h * rstd * gamma
    out = {"H": H if s["A"] is not None else None, "N": n.to(H.dtype) if "n" in case["out"] else None}
    if "q" in case["out"]:
        T, d = h.shape
        b = _groups(n, case["group"] or d)
        most = b.abs().amax(dim=2).clamp_min(SCALE_LEAST)
        out["Q"] = (b * (E4M3_MAX / most)[:, :, None]).clamp(-E4M3_MAX, E4M3_MAX).view(T, -1)[:, :d].to(E4M3)
        out["S"] = most / E4M3_MAX
    if case["op"] == "train":
        dn = s["dN"].float()
        dh = dn * gamma
        c = (dh * h).mean(dim=1, keepdim=True) * rstd * rstd * rstd
        out["dX"] = (s["dH"].float() + dh * rstd - h * c).to(H.dtype)
        out["dgamma"] = (dn * h * rstd).sum(dim=0)
    return out


def _own_norm(s):
    from paper_2604_11947_gb300 import resbm
    case = s["case"]
    resbm.resbm_add_rmsnorm_fwd(s["X"], s["A"], s["gamma"], EPS, s["H"], s["N"], s["Q"], s["S"], case["group"])
    out = {"H": s["H"], "N": s["N"]}
    if s["Q"] is not None:
        out["Q"], out["S"] = s["Q"], s["S"]
    if case["op"] == "train":
        resbm.resbm_rmsnorm_bwd(s["desc"], s["H"], s["gamma"], EPS, s["dN"], s["dH"], s["dX"], s["dgamma"], s["ws"])
        out["dX"], out["dgamma"] = s["dX"], s["dgamma"]
    return out


def _plain_gnorm(G):
    norm = G.float().square().sum(dtype=torch.float64).sqrt().float()
    return torch.stack((norm, (MAX_NORM / (norm + 1e-6)).clamp(max=1.0)))


def _plain_adamw(s, coef):
    h, t = HYPER, s["step"]
    bc1, bc2 = 1 - h["beta1"] ** t, 1 - h["beta2"] ** t
    g = s["G"].float()
    if coef is not None:
        g = g * coef
    if "Ms" in s:
        m = (s["M"].float().view(-1, BLOCK) * s["Ms"][:, None]).view(-1)
        v = (s["V"].float().view(-1, BLOCK) * s["Vs"][:, None]).view(-1).square_()
    else:
        m, v = s["M"], s["V"]
    # (each product rounded by itself: an 8-bit code next to a border does not depend on a fused multiply-add)
    m.mul_(h["beta1"]).add_(g * (1 - h["beta1"]))
    v.mul_(h["beta2"]).add_(g.square().mul_(1 - h["beta2"]))
    root = v.sqrt()
    if "Ms" in s:
        x, s["Ms"][:] = _code(m)
        s["M"].copy_(x.to(E4M3))
        x, s["Vs"][:] = _code(root)
        # a value above zero keeps a code above zero
        s["V"].copy_(torch.where(root > 0, x.clamp_min(E4M3_LEAST), 0.0).to(E4M3))
    w = s["master"] if "master" in s else s["W"].float()
    w.mul_(1 - h["lr"] * h["weight_decay"])
    w.addcdiv_(m, root.div_(math.sqrt(bc2)).add_(h["eps"]), value=-h["lr"] / bc1)
    s["W"].copy_(w)


def run(s):
    op = s["case"]["op"]
    if op in ("norm", "train"):
        return _own_norm(s) if own else _plain_norm(s)
    norm = None
    if own:
        from paper_2604_11947_gb300 import resbm
    if op == "gnorm" or s["case"]["clip"]:
        if own:
            norm = s["out"]
            resbm.resbm_grad_norm(s["plan"], MAX_NORM, norm, s["ws"])
        else:
            norm = _plain_gnorm(s["G"])
        if op == "gnorm":
            return {"norm": norm}
    s["step"] += 1
    if own:
        resbm.resbm_adamw_step(s["plan"], step=s["step"], grad_scale=None if norm is None else norm[1:], **HYPER)
    else:
        _plain_adamw(s, None if norm is None else norm[1])
    return {"norm": norm, **{k: s[k] for k in ("W", "master", "M", "Ms", "V", "Vs") if k in s}}


# ---- what a pass cannot do without ---------------------------------------------------------------
def work(case):
    size = {"bf16": 2, "f32": 4}
    if case["op"] in ("norm", "train"):
        T, d, e = case["T"], case["d"], size[case["dtype"]]
        groups = -(-d // (case["group"] or d))
        b = T * d * e + d * e                                      # X, gamma
        b += 2 * T * d * e if case["residual"] else 0              # A, H
        b += T * d * e if "n" in case["out"] else 0
        b += T * d + 4 * T * groups if "q" in case["out"] else 0
        flops = 6 * T * d
        if case["op"] == "train":
            b += 4 * T * d * e + d * e + 4 * d                     # H, dN, dH, dX, gamma, dgamma
            flops += 12 * T * d
        return {"bytes": b, "flops": flops}
    n = sum(_sizes(case))
    g = n * size[case["g"]]
    if case["op"] == "gnorm":
        return {"bytes": g + 8, "flops": 2 * n}
    b = g + 2 * n * size[case["w"]] + (8 * n if case["master"] else 0)
    if case["master"]:
        b -= n * size[case["w"]]                                   # the bf16 weight is written only
    blocks = sum(-(-k // BLOCK) for k in _sizes(case))
    b += 16 * n if case["bits"] == 32 else 4 * n + 16 * blocks
    # (with clipping the gradients are read twice: the step needs the norm of all of them)
    b += g if case["clip"] else 0
    return {"bytes": b, "flops": 14 * n}


# ---- the definitions in 64 bits --------------------------------------------------------------------
def _exact_norm(s):
    case = s["case"]
    X, gamma = s["X"].double(), s["gamma"].double()
    total = X if s["A"] is None else X + s["A"].double()
    out = {"H": None if s["A"] is None else total, "N": None}
    y = total.to(s["X"].dtype).double()   # the norm is taken of the sum as stored
    mean = (y * y).sum(dim=1, keepdim=True) / case["d"]
    scale = (mean + EPS).pow(-0.5)
    n = y * scale * gamma
    if "n" in case["out"]:
        out["N"] = n
    if "q" in case["out"]:
        g = case["group"] or case["d"]
        T, d = n.shape
        peak = torch.zeros(T, -(-d // g), dtype=torch.float64, device=n.device)
        index = (torch.arange(d, device=n.device) // g).expand(T, d)
        peak.scatter_reduce_(1, index, n.abs(), "amax")
        out["S"] = peak.clamp(min=SCALE_LEAST) / E4M3_MAX
        out["Q"] = n / out["S"].gather(1, index)
    if case["op"] == "train":
        dN = s["dN"].double()
        u = y * scale                                             # the normalised row
        along = ((dN * gamma) * u).sum(dim=1, keepdim=True) / case["d"]
        out["dX"] = s["dH"].double() + scale * (dN * gamma - u * along)
        out["dgamma"] = (dN * u).sum(dim=0)
    return out


def _exact_gnorm(s):
    norm = torch.linalg.vector_norm(s["G"].double())
    return torch.stack((norm, torch.minimum(torch.ones_like(norm), MAX_NORM / (norm + 1e-6))))


def _exact_adamw(s, norm):
    h, t = HYPER, s["step"] + 1
    g = s["G"].double() * (1.0 if norm is None else norm[1])
    wide = lambda k: s[k].double() * (s[k + "s"].double().repeat_interleave(BLOCK) if k + "s" in s else 1.0)
    m = h["beta1"] * wide("M") + (1 - h["beta1"]) * g
    v = h["beta2"] * (wide("V") ** 2 if "Vs" in s else wide("V")) + (1 - h["beta2"]) * g * g
    del g
    w = (s["master"] if "master" in s else s["W"]).double()
    mh, vh = m / (1 - h["beta1"] ** t), v / (1 - h["beta2"] ** t)
    w = w - h["lr"] * h["weight_decay"] * w - h["lr"] * mh / (vh.sqrt() + h["eps"])
    out = {"norm": norm, "W": w, "M": m, "V": v}
    if "master" in s:
        out["master"] = w
    if "Ms" in s:
        for k, x in (("M", m), ("V", v.sqrt())):
            x = x.view(-1, BLOCK)
            peak = x.abs().amax(dim=1).clamp(min=SCALE_LEAST) / E4M3_MAX
            out[k], out[k + "s"] = (x / peak[:, None]).view(-1), peak
    return out


def exact(case, seed):
    """What run() returns for these inputs, from the definitions in 64 bits (8-bit outputs in units of their scales, before
    their rounding)."""
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if case["op"] in ("norm", "train"):
        return _exact_norm(s)
    norm = _exact_gnorm(s) if case["op"] == "gnorm" or case["clip"] else None
    return {"norm": norm} if case["op"] == "gnorm" else _exact_adamw(s, norm)
