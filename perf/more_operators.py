"""Operators for learning from recorded choices and for orthogonalised updates, measured case by case.

  logprobs          log p of a given class per row, the entropy of the row's distribution and its most probable
                    classes:  z[n, v] = s (x[n] . w[v]) + offset[v],  log p[n, v] = z[n, v] - log sum_v exp(z[n, v])
  logprobs gradient the gradients in x and w for any upstream gradients of log p and entropy
  Muon step         momentum, orthogonalised by Newton-Schulz products, taken from the weights, over many matrices

A case is a dict of plain values. `prepare` makes what a program holds before the call, `run` is one pass: the
plain form (elementary torch operations in 32 bits) where `own` is false, the library's calls where it is true.
"""
import math

import torch

own = False

NEG = float("-inf")
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
DT = {"bf16": BF16, "f32": F32}
A, B, C = 3.4445, -4.7750, 2.0315   # the quintic that takes singular values of (0, 1] to about 1 in five steps
STEPS = 5


# ---------------------------------------------------------------------------------------------- cases
def _choice(name, op, dtype, rows, dim, classes, top, ignored=0.0, offset=False):
    return {"name": name, "op": op, "dtype": dtype, "rows": rows, "dim": dim, "classes": classes, "top": top,
            "ignored": ignored, "offset": offset}


def _muon(name, param, grad, layers, dim, wide, rank, nesterov=True):
    return {"name": name, "op": "muon", "param": param, "grad": grad, "layers": layers, "dim": dim, "wide": wide,
            "rank": rank, "nesterov": nesterov}


def listed():
    return [
        # one request answered from every class, with its eight best: latency and the read of w
        _choice("answer_one", "answer", "bf16", 1, 512, 50000, 8),
        # a request's fifty positions over an odd number of classes, some of them masked
        _choice("answer_ragged", "answer", "bf16", 50, 1856, 100003, 5, offset=True),
        # recorded choices of a batch scored under the present weights, with alternatives
        _choice("answer_batch", "answer", "bf16", 4096, 1856, 32000, 8, ignored=0.1),
        # a small model in float
        _choice("answer_float", "answer", "f32", 512, 160, 5000, 4),
        # one pass of learning from choices: a ragged last batch of a small model, padding rows, masked classes
        _choice("learn_ragged", "learn", "bf16", 333, 136, 1001, 0, ignored=0.3, offset=True),
        # the ordinary pass
        _choice("learn", "learn", "bf16", 4096, 1856, 32000, 0, ignored=0.05),
        # the largest: a long batch of positions, a wide model, a vocabulary of 2^17
        _choice("learn_large", "learn", "bf16", 8192, 4352, 131072, 0, ignored=0.05),
        # the matrices of the smallest model: latency
        _muon("muon_tiny", "f32", "f32", 2, 160, 32, 32),
        # odd sizes, bf16 weights without masters, rounded by chance, plain momentum
        _muon("muon_odd", "bf16", "bf16", 2, 1001, 333, 37, False),
        # a model of three attention layers, bf16 weights with float masters
        _muon("muon_small", "master", "f32", 3, 1856, 768, 256),
        # a wide stack of low rank, bf16 gradients
        _muon("muon_wide", "master", "bf16", 4, 4352, 512, 512),
        # the largest stack: four projections of rank 1024 over two wide layers
        _muon("muon_large", "master", "bf16", 2, 10624, 4096, 2048),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("answer", "learn", "muon"))
    if op == "muon":
        return _nameless(_muon("", rng.choice(("f32", "master", "bf16")), rng.choice(("f32", "bf16")),
                               rng.randint(1, 4), _log(rng, 16, 6000), _log(rng, 4, 2200), _log(rng, 4, 1100),
                               rng.random() < 0.7))
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    if dtype == "f32":
        rows, dim, classes = _log(rng, 1, 2000), 4 * _log(rng, 8, 128), _log(rng, 40, 16000)
    else:
        rows, dim, classes = _log(rng, 1, 8192), 8 * _log(rng, 8, 544), _log(rng, 100, 131072)
    top = 0 if op == "learn" else rng.choice((0, 1, 4, 8, 20))
    return _nameless(_choice("", op, dtype, rows, dim, classes, top, rng.choice((0.0, 0.05, 0.5)), rng.random() < 0.5))


def _nameless(case):
    del case["name"]
    return case


def _muon_shapes(case):
    return [s for _ in range(case["layers"]) for s in ((case["wide"], case["dim"]), (case["dim"], case["rank"]))]


# ------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if case["op"] == "muon":
        return _prepare_muon(case, g)
    rows, dim, classes, dt = case["rows"], case["dim"], case["classes"], DT[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    s = dict(case)
    s["x"] = normal(rows, dim).to(dt)
    s["w"] = (normal(classes, dim) * (3.0 / math.sqrt(dim))).to(dt)
    s["logit_scale"] = 0.75
    # choices of a heavy-tailed frequency; padding rows have label -1
    u = torch.rand(rows, generator=g, device="cuda", dtype=F64)
    s["labels"] = (classes * u ** 3).long().clamp_(0, classes - 1)
    s["offset"] = None
    if case["offset"]:
        # minus the log of a sampling frequency; the last hundredth of the classes is masked
        q = torch.arange(1, classes + 1, device="cuda", dtype=F32)
        s["offset"] = torch.log(q) * 0.5 - 0.5 * math.log(classes)
        masked = classes // 100
        if masked:
            s["offset"][classes - masked:] = NEG
            s["labels"].clamp_(max=classes - masked - 1)
    if case["ignored"]:
        s["labels"][torch.rand(rows, generator=g, device="cuda") < case["ignored"]] = -1
    if case["op"] == "learn":
        # minus advantage times importance ratio, and the weight of an entropy bonus that differs from row to row
        s["grad_logprob"] = normal(rows) / rows
        s["grad_entropy"] = -(torch.rand(rows, generator=g, device="cuda") * 0.1) / rows
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    """What a program keeps for its calls: a handle, result buffers and workspaces."""
    lib, rows, dim, classes, top = _handle(s["dtype"]), s["rows"], s["dim"], s["classes"], s["top"]
    forward, kept, grad, _ = lib.logprobs_workspace(rows, dim, classes, top)

    def buffer(n):
        return torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")

    s["lib"] = lib
    s["out"] = [torch.empty(rows, device="cuda") for _ in range(3)]
    s["top_ids"] = torch.empty(rows, top, dtype=torch.int64, device="cuda") if top else None
    s["top_logprob"] = torch.empty(rows, top, device="cuda") if top else None
    learn = s["op"] == "learn"
    s["stats"] = torch.empty(rows, 4, device="cuda") if learn else None
    s["kept"] = buffer(kept) if learn else None
    s["scratch"] = buffer(max(forward, grad) if learn else forward)
    if learn:
        s["grad_x"], s["grad_w"] = torch.empty_like(s["x"]), torch.empty_like(s["w"])


def _prepare_muon(case, g):
    s = dict(case)
    s.update(lr=1e-3, momentum=0.95, seed=1234567)
    s["tensors"] = []
    for rows, cols in _muon_shapes(case):
        short = min(rows, cols)
        # a gradient's singular values fall off: its directions are of very different sizes
        size = (torch.arange(1, short + 1, device="cuda", dtype=F32) ** -0.5) * (0.1 / short)

        def falling():
            left = torch.randn(rows, short, generator=g, device="cuda") * size
            return left @ torch.randn(short, cols, generator=g, device="cuda")

        p = torch.randn(rows, cols, generator=g, device="cuda") * 0.05
        t = {"master": p if case["param"] == "master" else None,
             "param": p if case["param"] == "f32" else p.to(BF16),
             "grad": falling().to(DT[case["grad"]]), "m": falling() * 0.5, "weight_decay": 0.01,
             # the size of an update's elements, whatever the matrix's shape: that of AdamW's
             "scale": 0.2 * math.sqrt(max(rows, cols))}
        s["tensors"].append(t)
    if own:
        from paper_2402_06859_amd import rdcn
        s["lib"] = _handle("bf16")
        s["list"] = rdcn.muon_tensors(s["tensors"])
        s["scratch"] = torch.empty(max(256, s["lib"].muon_workspace(s["list"])), dtype=torch.uint8, device="cuda")
    return s


_handles = {}


def _handle(dtype):
    if dtype not in _handles:
        from paper_2402_06859_amd import rdcn
        _handles[dtype] = rdcn.Rdcn(rdcn.make_config(8192, 4, 16, 32, 8, 1, 25, 25, 600, dtype=dtype))
    return _handles[dtype]


# ---------------------------------------------------------------------------------------- one pass
def run(s):
    if s["op"] == "muon":
        return _own_muon(s) if own else _plain_muon(s)
    if own:
        return _own_choice(s)
    return _plain_answer(s) if s["op"] == "answer" else _plain_learn(s)


def _own_choice(s):
    lib, (logprob, entropy, lse) = s["lib"], s["out"]
    size = (s["rows"], s["dim"], s["classes"])
    given = (s["x"], s["w"], s["offset"], s["labels"], s["logit_scale"])
    lib.logprobs_forward(*size, *given, logprob, entropy, lse, s["scratch"], top=s["top"], top_ids=s["top_ids"],
                         top_logprob=s["top_logprob"], stats=s["stats"], kept=s["kept"])
    if s["op"] == "answer":
        return {"logprob": logprob, "entropy": entropy, "lse": lse, "top_ids": s["top_ids"],
                "top_logprob": s["top_logprob"]}
    lib.logprobs_grad(*size, *given, s["stats"], s["grad_logprob"], s["grad_entropy"], s["grad_x"], s["grad_w"],
                      s["scratch"], kept=s["kept"])
    return {"logprob": logprob, "entropy": entropy, "lse": lse, "grad_x": s["grad_x"], "grad_w": s["grad_w"]}


def _plain_logits(s):
    z = (s["x"].float() @ s["w"].float().t()) * s["logit_scale"]
    return z if s["offset"] is None else z + s["offset"]


def _plain_values(s, z):
    """log p of the labels, entropies, and each row's log sum and its logits less that."""
    top = z.amax(1, keepdim=True)
    lse = torch.exp(z - top).sum(1, keepdim=True).log() + top
    logp = z - lse
    entropy = -(torch.exp(logp) * torch.where(logp == NEG, 0.0, logp)).sum(1)
    given = logp.gather(1, s["labels"].clamp(min=0)[:, None])[:, 0]
    return torch.where(s["labels"] >= 0, given, 0.0), entropy, lse[:, 0], logp


def _plain_answer(s):
    z = _plain_logits(s)
    logprob, entropy, lse, logp = _plain_values(s, z)
    out = {"logprob": logprob, "entropy": entropy, "lse": lse, "top_ids": None, "top_logprob": None}
    if s["top"]:
        # near ties are decided in 64 bits, among somewhat more candidates than are wanted
        cand = z.topk(min(s["classes"], s["top"] + 8), 1).indices.sort(1).values
        z64 = (s["w"][cand].double() * s["x"].double()[:, None]).sum(2) * s["logit_scale"]
        if s["offset"] is not None:
            z64 += s["offset"].double()[cand]
        best = z64.sort(dim=1, descending=True, stable=True).indices[:, :s["top"]]
        out["top_ids"] = cand.gather(1, best)
        out["top_logprob"] = logp.gather(1, out["top_ids"])
    return out


def _plain_learn(s):
    z = _plain_logits(s)
    logprob, entropy, lse, logp = _plain_values(s, z)
    kept = (s["labels"] >= 0).float()
    g, h = (s["grad_logprob"] * kept)[:, None], (s["grad_entropy"] * kept)[:, None]
    p = torch.exp(logp)
    # d log p_y / dz = onehot - p,  dH / dz = -p (log p + H)
    d = p * (-g - h * (torch.where(logp == NEG, 0.0, logp) + entropy[:, None]))
    d.scatter_add_(1, s["labels"].clamp(min=0)[:, None], g)
    d *= s["logit_scale"]
    return {"logprob": logprob, "entropy": entropy, "lse": lse, "grad_x": (d @ s["w"].float()).to(s["x"].dtype),
            "grad_w": (d.t() @ s["x"].float()).to(s["w"].dtype)}


def _own_muon(s):
    s["lib"].muon_step(s["list"], s["scratch"], lr=s["lr"], momentum=s["momentum"], nesterov=s["nesterov"],
                       coefficients=(A, B, C), steps=STEPS, stochastic=True, seed=s["seed"])
    return [{"param": t["param"], "master": t["master"], "m": t["m"]} for t in s["tensors"]]


def _plain_muon(s):
    return [_plain_step(s, t, i) for i, t in enumerate(s["tensors"])]


def _plain_step(s, t, ordinal):
    mu = s["momentum"]
    g = t["grad"].float() * (1.0 - mu)
    m = t["m"] * mu + g
    u = m * mu + g if s["nesterov"] else m
    tall = u.shape[0] > u.shape[1]
    x = u.t() if tall else u
    x = x / x.double().square().sum().sqrt().float()
    x = _plain_round(_plain_round(_plain_round(_plain_round(_plain_round(x)))))
    o = x.t() if tall else x
    p = t["master"] if t["master"] is not None else t["param"].float()
    p = p * (1.0 - s["lr"] * t["weight_decay"]) - o * (s["lr"] * t["scale"])
    t["m"].copy_(m)
    if t["master"] is not None:
        t["master"].copy_(p)
        t["param"].copy_(p)
    elif t["param"].dtype == BF16:
        # by chance: the bits below a bf16's are the probability of rounding up
        bits = (p.view(torch.int32).long() & 0xFFFFFFFF) + _chance(p.numel(), ordinal, s["seed"]).view(p.shape)
        bits = (bits >> 16) << 16
        t["param"].copy_(torch.where(bits >= 1 << 31, bits - (1 << 32), bits).to(torch.int32).view(F32))
    else:
        t["param"].copy_(p)
    return {"param": t["param"], "master": t["master"], "m": t["m"]}


def _plain_round(x):
    a = x @ x.t()
    return A * x + (B * a + C * (a @ a)) @ x


def _chance(n, ordinal, seed):
    """16 bits for every element of a tensor, random inputs of the rounding (fmix32, the finalizer of MurmurHash3)."""
    h = torch.arange(n, device="cuda", dtype=torch.int64) & 0xFFFFFFFF
    h = h ^ ((seed + 0x9E3779B9 * (ordinal + 1)) & 0xFFFFFFFF)
    h = ((h ^ (h >> 16)) * 0x85EBCA6B) & 0xFFFFFFFF
    h = ((h ^ (h >> 13)) * 0xC2B2AE35) & 0xFFFFFFFF
    h = h ^ (h >> 16)
    return ((h * 0x85EBCA6B) & 0xFFFFFFFF) >> 16


# ------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["op"] == "muon":
        bytes_, flops = 0, 0
        for rows, cols in _muon_shapes(case):
            n, m, r = rows * cols, min(rows, cols), max(rows, cols) / min(rows, cols)
            bytes_ += n * ({"f32": 8, "bf16": 4, "master": 10}[case["param"]] + 8 + {"f32": 4, "bf16": 2}[case["grad"]])
            # the products on the Gram matrix, symmetric ones counted half: X X^T once, for five steps A^2, T A, T (T A) and
            # T P where they are needed (17 in all), and P X
            flops += min(17 + 3 * r, 5 * (3 * r + 1)) * m ** 3
        return {"bytes": bytes_, "flops": flops}
    rows, dim, classes, e = case["rows"], case["dim"], case["classes"], 2 if case["dtype"] == "bf16" else 4
    io = (rows + classes) * dim * e + rows * 20 + rows * case["top"] * 12 + (4 * classes if case["offset"] else 0)
    if case["op"] == "answer":
        return {"bytes": io, "flops": 2 * rows * dim * classes}
    # logits, the gradient in x and the gradient in w: one product each
    return {"bytes": io + rows * 8 + (rows + classes) * dim * e, "flops": 6 * rows * dim * classes}


# ------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "muon":
        return _exact_muon(s)
    x, w, y = s["x"].double(), s["w"].double(), s["labels"]
    off = 0.0 if s["offset"] is None else s["offset"].double()
    rows, top, learn = case["rows"], case["top"], case["op"] == "learn"
    out = {k: torch.zeros(rows, dtype=F64, device="cuda") for k in ("logprob", "entropy", "lse")}
    ids = torch.zeros(rows, top, dtype=torch.int64, device="cuda")
    best = torch.zeros(rows, top, dtype=F64, device="cuda")
    gx, gw = (torch.zeros_like(x), torch.zeros_like(w)) if learn else (None, None)
    part = max(1, min(rows, 100_000_000 // case["classes"]))
    for at in range(0, rows, part):
        here = slice(at, min(rows, at + part))
        xs, ys = x[here], y[here]
        lp = torch.log_softmax(s["logit_scale"] * torch.mm(xs, w.t()) + off, 1)
        p = lp.exp()
        seen = lp.masked_fill(lp == NEG, 0.0)
        h = -(p * seen).sum(1)
        known = torch.nonzero(ys >= 0)[:, 0]
        out["logprob"][at + known] = lp[known, ys[known]]
        out["entropy"][here] = h
        out["lse"][here] = torch.logsumexp(s["logit_scale"] * torch.mm(xs, w.t()) + off, 1)
        if top:
            v, i = torch.sort(lp, dim=1, descending=True, stable=True)
            best[here], ids[here] = v[:, :top], i[:, :top]
        if learn:
            ga, ha = torch.zeros(2, len(ys), dtype=F64, device="cuda")
            ga[known] = s["grad_logprob"].double()[at + known]
            ha[known] = s["grad_entropy"].double()[at + known]
            d = -(p * seen.add_(h[:, None]).mul_(ha[:, None]).add_(ga[:, None]))
            d[known, ys[known]] += ga[known]
            d *= s["logit_scale"]
            gx[here] = torch.mm(d, w)
            gw += torch.mm(d.t(), xs)
    if learn:
        return {**out, "grad_x": gx, "grad_w": gw}
    return {**out, "top_ids": ids if top else None, "top_logprob": best if top else None}


def _exact_muon(s):
    out = []
    for t in s["tensors"]:
        g, mu = t["grad"].double(), s["momentum"]
        m = torch.lerp(g, t["m"].double(), mu)
        x = torch.lerp(g, m, mu) if s["nesterov"] else m.clone()
        x /= torch.linalg.matrix_norm(x)
        for _ in range(STEPS):
            # the polynomial on the shorter side's Gram matrix, from whichever side that is
            if x.shape[0] <= x.shape[1]:
                q = torch.mm(x, x.mT)
                x = torch.mm(A * torch.eye(len(q), dtype=F64, device="cuda") + B * q + C * torch.mm(q, q), x)
            else:
                q = torch.mm(x.mT, x)
                x = torch.mm(x, A * torch.eye(len(q), dtype=F64, device="cuda") + B * q + C * torch.mm(q, q))
        p0 = (t["param"] if t["master"] is None else t["master"]).double()
        p = p0 - s["lr"] * (t["weight_decay"] * p0 + t["scale"] * x)
        by_chance = t["master"] is None and t["param"].dtype == BF16
        out.append({"param": None if by_chance else p, "master": None if t["master"] is None else p, "m": m})
    return out
