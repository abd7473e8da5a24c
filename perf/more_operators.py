"""Timed cases of the vocabulary's operators: what the first and the last stage of a pipeline have the library do with the
embedding table and the output head.

Every case is a dict with an "op":

  ce       resbm_linear_ce_fwd: the cross entropy of tokens' hidden states X (T x d) against a head W (V x d), without storing
           the logits X . W^T; with "train", resbm_linear_ce_bwd after it: dX and dW of the incoming gradient of the losses
  distill  resbm_distill_fwd, and with "train" resbm_distill_bwd: the divergence from a teacher's K largest logits at a
           temperature, over the same logits
  embed    resbm_embed_fwd: rows of the table times a scale; with "train", resbm_embed_bwd: the table's gradient

The plain forms here are elementary torch operations in fp32 (the library's own calls run where `own` is true).
"""
import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
MOST_PRODUCT = 4096 * 131072 * 4096   # T V d of the largest listed case
MOST_LOGITS = 1 << 31                 # T V of a drawn case: 8.6 GB a copy in the plain form
MOST_TABLE = 250_002 * 1003           # V d of the largest listed table
MOST_ROWS = 65536 * 2048              # T d of a drawn lookup


def _loss(name, op, T, V, d, **kw):
    case = {"name": name, "op": op, "T": T, "V": V, "d": d, "dtype": "bf16", "train": False, "ignored": 0.0, "weights": False,
            "pad": 0, "K": 0, "temperature": 1.0}
    case.update(kw)
    return case


def _embed(name, T, V, d, **kw):
    case = {"name": name, "op": "embed", "T": T, "V": V, "d": d, "dtype": "bf16", "train": False, "scale": 1.0, "padding": 0.0}
    case.update(kw)
    return case


def listed():
    return [
        # The score of one position: the smallest call, the head read once.
        _loss("ce_token", "ce", 1, 32000, 2048),
        # A held-out batch of odd sizes, scored (no gradient).
        _loss("ce_score_ragged", "ce", 777, 50001, 1000, ignored=0.05),
        # The convergence comparison's batch (16 x 256 tokens, 256 words, d = 512), forward and backward.
        _loss("ce_train_convergence", "ce", 4096, 256, 512, train=True, ignored=1 / 256),
        # The simulated pipeline's last stage: batch 8 x seq 2048, the last position of every sequence without a label.
        _loss("ce_train_pipeline", "ce", 16384, 32000, 2048, train=True, ignored=1 / 2048),
        # Fine-tuning: prompts and padding carry no label, the tokens weights of their own.
        _loss("ce_train_masked", "ce", 8192, 32000, 2048, train=True, ignored=0.6, weights=True),
        # A larger vocabulary and the headline workload's width, a microbatch.
        _loss("ce_train_wide", "ce", 4096, 131072, 4096, train=True),
        # A model in fp32.
        _loss("ce_train_f32", "ce", 2048, 8000, 768, dtype="f32", train=True, ignored=0.02),
        # A microbatch of the pipeline against a teacher's 64 largest logits at temperature 2.
        _loss("distill_train", "distill", 4096, 32000, 2048, train=True, K=64, temperature=2.0),
        # Odd sizes, a few entries a token, some of them missing, hidden states that are a slice of a wider buffer.
        _loss("distill_ragged", "distill", 333, 20011, 1000, train=True, ignored=0.1, weights=True, pad=24, K=7),
        # Eight sequences' next tokens: latency.
        _embed("embed_token", 8, 32000, 4096, scale=64.0),
        # The pipeline's first stage, forward and backward.
        _embed("embed_train_pipeline", 16384, 32000, 2048, train=True),
        # A large table of an odd width in fp32, two fifths of the tokens padding.
        _embed("embed_train_padded", 65536, 250_002, 1003, dtype="f32", train=True, scale=31.67, padding=0.4),
    ]


def draw(rng):
    log = lambda a, b: int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))
    op = rng.choice(("ce", "ce", "distill", "embed"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if op == "embed":
        d = log(64, 4096)
        V = log(64, min(250_002, MOST_TABLE // d))
        case = {"op": op, "T": log(1, min(65536, MOST_ROWS // d)), "V": V, "d": d, "dtype": dtype, "train": rng.random() < 0.7,
                "scale": rng.choice((1.0, math.sqrt(d))), "padding": rng.choice((0.0, 0.0, 0.3))}
        return case
    d = log(64, 4096)
    if rng.random() < 0.6:
        d = d // 8 * 8
    V = log(64, 131072)
    T = log(1, max(1, min(16384, MOST_LOGITS // V, MOST_PRODUCT // (4 if dtype == "f32" else 1) // (V * d))))
    case = {"op": op, "T": T, "V": V, "d": d, "dtype": dtype, "train": rng.random() < 0.7, "ignored": rng.choice((0.0, 0.01, 0.5)),
            "weights": rng.random() < 0.4, "pad": rng.choice((0, 0, 8, 5)), "K": 0, "temperature": 1.0}
    if op == "distill":
        case["K"], case["temperature"] = min(V, log(1, 128)), rng.choice((1.0, 1.0, 2.0, 0.7))
    return case


# ---- inputs --------------------------------------------------------------------------------------
def _gen(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _zipf(n, V, gen):
    """n token ids whose frequencies fall with their rank."""
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    return (torch.exp(u * math.log(V + 1)) - 1).long().clamp_(0, V - 1)


def _prepare_loss(case, gen):
    T, V, d, K, dt = case["T"], case["V"], case["d"], case["K"], DT[case["dtype"]]
    normal = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")
    s = {"case": case, "tau": case["temperature"]}
    std = 1.0 / math.sqrt(d)                                     # logits of about one
    W = normal(V, d).mul_(std)
    without = torch.randperm(T, generator=gen, device="cuda")[:int(T * case["ignored"])]
    if case["op"] == "ce":
        label = _zipf(T, V, gen)
        aim = label
        s["labels"] = label.clone()
        s["labels"][without] = -100
    else:
        # K places of the vocabulary in no order, and the teacher's logits there, falling from the first on
        step = 1 + (torch.rand(T, 1, generator=gen, device="cuda") * (V // K)).long().clamp_(max=V // K - 1)
        index = (_zipf(T, V, gen)[:, None] + step * torch.arange(K, device="cuda")) % V
        fall = -torch.log(torch.rand(T, K, generator=gen, device="cuda").clamp_min(1e-6)) * 0.3
        teacher = 12.0 - fall.cumsum(dim=1)
        aim = index[:, 0]
        order = torch.randperm(K, generator=gen, device="cuda")
        index, teacher = index[:, order].contiguous(), teacher[:, order].to(dt).contiguous()
        if K > 4:                                                # fewer than K for some tokens
            index[::5, K - 2] = -1
        index[without] = -1
        s["index"], s["teacher"] = index, teacher
    # hidden states that know something of what follows: from nothing to near certainty
    X = normal(T, d + case["pad"])
    X[:, :d] += W[aim] * (torch.rand(T, 1, generator=gen, device="cuda") * 14.0)
    s["X"], s["W"] = X.to(dt)[:, :d], W.to(dt)
    new = lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device="cuda")
    s["loss"], s["lse"] = new(T), new(T)
    if case["train"]:
        n = T - without.numel()
        s["dloss"] = torch.full((1,), 1.0 / max(n, 1), device="cuda")
        if case["weights"]:
            s["dloss"] = torch.rand(T, generator=gen, device="cuda") * (2.0 / max(n, 1))
        s["dX"], s["dW"] = new(T, d, dtype=dt), new(V, d, dtype=dt)
    if own:
        from paper_2604_11947_gb300 import resbm
        kinds = {("ce", False): resbm.RESBM_VOCAB_CE_FWD, ("ce", True): resbm.RESBM_VOCAB_CE_BWD,
                 ("distill", False): resbm.RESBM_VOCAB_DISTILL_FWD, ("distill", True): resbm.RESBM_VOCAB_DISTILL_BWD}
        need = max(resbm.resbm_vocab_workspace_bytes(kinds[case["op"], b], T, V, d, case["dtype"], K) for b in {False, case["train"]})
        s["ws"] = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    return s


def _prepare_embed(case, gen):
    T, V, d, dt = case["T"], case["V"], case["d"], DT[case["dtype"]]
    s = {"case": case, "padding": -1}
    s["ids"] = _zipf(T, V, gen)
    if case["padding"]:
        s["padding"] = V // 2
        s["ids"][torch.rand(T, generator=gen, device="cuda") < case["padding"]] = s["padding"]
    s["table"] = (0.02 * torch.randn(V, d, generator=gen, device="cuda")).to(dt)
    s["out"] = torch.empty(T, d, dtype=dt, device="cuda")
    if case["train"]:
        s["dout"] = (1e-3 * torch.randn(T, d, generator=gen, device="cuda")).to(dt)
        s["dtable"] = torch.empty(V, d, dtype=dt, device="cuda")
        if own:
            from paper_2604_11947_gb300 import resbm
            s["ws"] = resbm.vocab_workspace(resbm.RESBM_VOCAB_EMBED_BWD, T, V, d, case["dtype"])
    return s


def prepare(case, seed):
    return (_prepare_embed if case["op"] == "embed" else _prepare_loss)(case, _gen(seed))


# ---- one pass ------------------------------------------------------------------------------------
def _plain_targets(s):
    """The places of a token's targets, their weights, and which tokens have any."""
    if "labels" in s:
        there = s["labels"] >= 0
        return s["labels"].clamp_min(0)[:, None], there.float()[:, None], there
    there = s["index"] >= 0
    t = torch.where(there, s["teacher"].float() / s["tau"], -torch.inf)
    some = there.any(dim=1)
    q = torch.exp(t - torch.where(some, t.amax(dim=1), 0.0)[:, None])
    q = q / torch.where(some, q.sum(dim=1), 1.0)[:, None]
    return s["index"].clamp_min(0), q, some


def _plain_loss(s):
    case, tau = s["case"], s["tau"]
    at, q, some = _plain_targets(s)
    x, w = s["X"].float(), s["W"].float()
    z = x @ w.t()
    if tau != 1.0:
        z /= tau
    most = z.amax(dim=1)
    lse = most + torch.log(torch.exp(z - most[:, None]).sum(dim=1))
    loss = lse - (q * z.gather(1, at)).sum(dim=1)
    if case["op"] == "distill":
        loss = tau * tau * (loss + (q * torch.where(q > 0, q, 1.0).log()).sum(dim=1))
    out = {"loss": torch.where(some, loss, 0.0), "lse": torch.where(some, lse, 0.0)}
    if case["train"]:
        g = torch.where(some, s["dloss"] * tau, 0.0)
        dz = torch.exp(z.sub_(lse[:, None])).mul_(g[:, None])
        dz.scatter_add_(1, at, -(q * g[:, None]))
        out["dX"], out["dW"] = (dz @ w).to(s["X"].dtype), (dz.t() @ x).to(s["W"].dtype)
    return out


def _own_loss(s):
    from paper_2604_11947_gb300 import resbm
    X, W, loss, lse, ws, train = s["X"], s["W"], s["loss"], s["lse"], s["ws"], s["case"]["train"]
    if s["case"]["op"] == "ce":
        resbm.resbm_linear_ce_fwd(X, W, s["labels"], loss, lse, ws)
        if train:
            resbm.resbm_linear_ce_bwd(X, W, s["labels"], lse, s["dloss"], s["dX"], s["dW"], ws)
    else:
        resbm.resbm_distill_fwd(X, W, s["index"], s["teacher"], s["tau"], loss, lse, ws)
        if train:
            resbm.resbm_distill_bwd(X, W, s["index"], s["teacher"], s["tau"], lse, s["dloss"], s["dX"], s["dW"], ws)
    return {"loss": loss, "lse": lse, **({"dX": s["dX"], "dW": s["dW"]} if train else {})}


def _plain_embed(s):
    case, ids = s["case"], s["ids"]
    out = {"out": (s["table"][ids].float() * case["scale"]).to(s["table"].dtype)}
    if case["train"]:
        rows = torch.where((ids != s["padding"])[:, None], s["dout"].float(), 0.0)
        total = torch.zeros(case["V"], case["d"], device="cuda").index_add_(0, ids, rows)
        out["dtable"] = (total * case["scale"]).to(s["table"].dtype)
    return out


def _own_embed(s):
    from paper_2604_11947_gb300 import resbm
    case = s["case"]
    resbm.resbm_embed_fwd(s["ids"], s["table"], case["scale"], s["out"])
    out = {"out": s["out"]}
    if case["train"]:
        resbm.resbm_embed_bwd(s["ids"], s["dout"], case["scale"], s["dtable"], s["ws"], padding=s["padding"])
        out["dtable"] = s["dtable"]
    return out


def run(s):
    if s["case"]["op"] == "embed":
        return _own_embed(s) if own else _plain_embed(s)
    return _own_loss(s) if own else _plain_loss(s)


# ---- what a pass cannot do without ---------------------------------------------------------------
def work(case):
    T, V, d, e = case["T"], case["V"], case["d"], SIZE[case["dtype"]]
    if case["op"] == "embed":
        n = T - int(T * case["padding"])
        b, flops = 8 * T + (min(T, V) + T) * d * e, T * d
        if case["train"]:
            b += 8 * T + (n + V) * d * e
            flops += 2 * n * d
        return {"bytes": b, "flops": flops}
    n = T - int(T * case["ignored"])                             # (tokens without a target cost nothing)
    targets = 8 * T if case["op"] == "ce" else (8 + e) * T * case["K"]
    b = (n + V) * d * e + targets + 8 * T
    if case["train"]:
        b += (T + V) * d * e + 4 * T                             # dX, dW, the losses' gradient
    return {"bytes": b, "flops": (6 if case["train"] else 2) * n * V * d}


# ---- the definitions in 64 bits --------------------------------------------------------------------
def _exact_loss(s):
    case, tau = s["case"], s["tau"]
    T, V = case["T"], case["V"]
    X, W = s["X"].double(), s["W"].double()
    goal = torch.zeros(T, V, dtype=torch.float64, device="cuda")   # the distribution that the student is held against
    if case["op"] == "ce":
        rows = torch.nonzero(s["labels"] >= 0)[:, 0]
        goal[rows, s["labels"][rows]] = 1.0
        self_entropy = torch.zeros(T, dtype=torch.float64, device="cuda")
    else:
        weight = torch.softmax(torch.where(s["index"] >= 0, s["teacher"].double() / tau, -torch.inf), dim=1)
        weight = torch.nan_to_num(weight, nan=0.0)
        goal.scatter_add_(1, s["index"].clamp(min=0), weight)
        self_entropy = torch.xlogy(weight, weight).sum(dim=1)
    held = goal.sum(dim=1) > 0.5
    logits = (X @ W.t()) / tau
    norm = torch.logsumexp(logits, dim=1)
    loss = tau * tau * (self_entropy + norm - (goal * logits).sum(dim=1))
    out = {"loss": loss * held, "lse": norm * held}
    if case["train"]:
        slope = (torch.softmax(logits, dim=1) - goal) * (s["dloss"].double() * tau * held)[:, None]
        out["dX"], out["dW"] = slope @ W, slope.t() @ X
    return out


def _exact_embed(s):
    case = s["case"]
    out = {"out": torch.nn.functional.embedding(s["ids"], s["table"].double()) * case["scale"]}
    if case["train"]:
        keep = s["ids"] != s["padding"]
        out["dtable"] = torch.zeros(case["V"], case["d"], dtype=torch.float64, device="cuda")
        out["dtable"].index_put_((s["ids"][keep],), s["dout"][keep].double() * case["scale"], accumulate=True)
    return out


def exact(case, seed):
    """What run() returns for these inputs, from the definitions in 64 bits."""
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return _exact_embed(s) if case["op"] == "embed" else _exact_loss(s)
