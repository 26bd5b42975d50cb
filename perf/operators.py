"""The operators at the end of a network -- layer norm, log probabilities, distillation -- as cases that can be timed and
compared.

`own` chooses what `run` computes with: False, the operators in plain torch (32-bit arithmetic whatever the inputs' type,
one rounding at the end); True, the calls that a program makes of the library through the binding.  Sizes are those of the
CaffeNet-shaped network (batch 256, 4096 and 9216 features, 1000 classes) or generic ones: vocabularies of 2^16 and 2^17,
odd counts of rows and classes, rows whose pitch is larger than their length.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5


def listed():
    return [
        # One image's or token's features, evaluated: nothing but latency.
        norm("norm forward f32 1x4096", "forward", 1, 4096, "f32"),
        # The features in front of the first fully connected layer, 256 x 6 x 6 an image, in a training step.
        norm("norm train bf16 256x9216", "train", 256, 9216, "bf16"),
        # Odd rows of a matrix whose pitch is larger than its width.
        norm("norm train f32 1023x1001", "train", 1023, 1001, "f32", 1024),
        # A long batch of token features, in a training step.
        norm("norm train bf16 16384x4096", "train", 16384, 4096, "bf16"),
        # What one decoded token is answered with: its own score and twenty alternatives of a vocabulary of 2^17.
        logprob("logprob forward bf16 1x131072 top20", "forward", 1, 131072, "bf16", top=20),
        # The evaluation of one batch of the CaffeNet-shaped network: the labels' scores and the five best classes.
        logprob("logprob forward f32 256x1000 top5", "forward", 256, 1000, "f32", top=5),
        # Policy training on sampled tokens: scores, entropies and their gradient; an odd vocabulary without row padding.
        logprob("logprob train bf16 2047x50021", "train", 2047, 50021, "bf16"),
        # A long prompt scored at every position, as a teacher's top entries are written out.
        logprob("logprob forward bf16 2048x131072 top32", "forward", 2048, 131072, "bf16", top=32, masked=0.02),
        # One batch of the CaffeNet-shaped network taught by ten classes a row and by the labels, both directions at once.
        distill("distill both f32 256x1000 k10", "both", 256, 1000, "f32", 10, 0.7, 4.0),
        # Few long rows, evaluated: a held-out loss over one short sequence.
        distill("distill forward bf16 48x131072 k50", "forward", 48, 131072, "bf16", 50, 1.0, 1.0),
        # The two directions on their own, odd sizes in fp32.
        distill("distill split f32 1021x32003 k31", "split", 1021, 32003, "f32", 31, 1.0, 2.0, 32064),
        # The largest step: loss and gradient over a vocabulary of 2^16.
        distill("distill both bf16 4096x65536 k64", "both", 4096, 65536, "bf16", 64, 0.5, 2.0),
    ]


def norm(name, way, rows, width, dtype, ld=0):
    return {"name": name, "kind": "norm", "way": way, "rows": rows, "width": width, "dtype": dtype, "ld": max(ld, width)}


def logprob(name, way, rows, classes, dtype, top=0, masked=0.0, temperature=1.0, ld=0):
    return {"name": name, "kind": "logprob", "way": way, "rows": rows, "width": classes, "dtype": dtype, "top": top, "masked": masked,
            "temperature": temperature, "ld": max(ld, classes)}


def distill(name, way, rows, classes, dtype, kept, alpha, temperature, ld=0):
    return {"name": name, "kind": "distill", "way": way, "rows": rows, "width": classes, "dtype": dtype, "kept": kept, "alpha": alpha,
            "temperature": temperature, "ld": max(ld, classes)}


# ---------------------------------------------------------------------------------------------- the ranges
def spread(rng, lo, hi):
    """A whole number between lo and hi, spread over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """Rows of 1 to 16384, widths of 16 to 2^17, at most the largest listed cases' elements of each kind."""
    kind, dtype = rng.choice(["norm", "logprob", "distill"]), rng.choice(["bf16", "f32"])
    width = spread(rng, 16, 16384) if kind == "norm" else spread(rng, 100, 131072)
    most = (16384 * 4096 if kind == "norm" else 2048 * 131072) // (1 if dtype == "bf16" else 2)
    rows = spread(rng, 1, min(16384, most // width))
    ld = rng.choice([width, width, (width + 63) // 64 * 64])
    if kind == "norm":
        case = norm("", rng.choice(["forward", "train", "train"]), rows, width, dtype, ld)
    elif kind == "logprob":
        case = logprob("", rng.choice(["forward", "forward", "train"]), rows, width, dtype, rng.choice([0, 1, 5, 20, 40]),
                       rng.choice([0.0, 0.0, 0.1]), rng.choice([1.0, 0.7, 1.3]), ld)
    else:
        case = distill("", rng.choice(["both", "both", "split", "forward"]), rows, width, dtype, spread(rng, 1, 64),
                       rng.choice([1.0, 0.5, 0.9]), rng.choice([1.0, 2.0, 4.0]), ld)
    del case["name"]
    return case


# ---------------------------------------------------------------------------------------------- state
def matrix(g, case, sigma=1.0, mean=0.0):
    """[rows][width] of a matrix with the case's pitch."""
    full = torch.randn((case["rows"], case["ld"]), generator=g, device="cuda", dtype=torch.float32)
    return full.mul_(sigma).add_(mean).to(TYPES[case["dtype"]])[:, :case["width"]]


def empty(case):
    return torch.empty((case["rows"], case["ld"]), dtype=TYPES[case["dtype"]], device="cuda")[:, :case["width"]]


def floats(*shape):
    return torch.empty(shape, dtype=torch.float32, device="cuda")


def prepare(case, seed):
    """Inputs, and the output buffers that a program which makes this call again and again keeps."""
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    rows, width = case["rows"], case["width"]
    st = dict(case)
    train = case["way"] != "forward"
    if case["kind"] == "norm":
        st["x"] = matrix(g, case, 1.5, 0.3)
        st["gamma"] = 1.0 + 0.1 * torch.randn(width, generator=g, device="cuda")
        st["beta"] = 0.1 * torch.randn(width, generator=g, device="cuda")
        st["out"] = {"y": empty(case)}
        if train:
            st["dy"] = matrix(g, case, 2.0 ** -6)
            st["out"].update(mean=floats(rows), rstd=floats(rows), dx=empty(case), dgamma=floats(width), dbeta=floats(width))
        return st
    x = st["logits"] = matrix(g, case, 2.5)
    if case["kind"] == "logprob":
        if case["masked"]:  # classes that are not allowed
            x.masked_fill_(torch.rand((1, width), generator=g, device="cuda") < case["masked"], -math.inf)
        st["targets"] = torch.randint(0, width, (rows,), generator=g, device="cuda")
        st["out"] = {"logprob": floats(rows), "entropy": floats(rows), "stats": floats(rows, 2)}
        if case["top"]:
            st["out"].update(top_index=torch.empty((rows, case["top"]), dtype=torch.int64, device="cuda"), top_logprob=floats(rows, case["top"]))
        if train:
            st["dlogprob"] = torch.randn(rows, generator=g, device="cuda") / rows       # advantages
            st["dentropy"] = torch.full((rows,), -0.01 / rows, device="cuda")
            st["out"]["dlogits"] = empty(case)
        return st
    teacher = x.float() * 0.8
    teacher += torch.randn(x.shape, generator=g, device="cuda")
    st["teacher_logits"], st["teacher_index"] = (t.contiguous() for t in teacher.topk(case["kept"], dim=1))
    del teacher
    # rows that were stored with fewer entries than the matrix has room for, and rows without a label
    short = torch.rand((rows, 1), generator=g, device="cuda") < 0.1
    st["teacher_index"][short & (torch.arange(case["kept"], device="cuda") >= max(1, case["kept"] // 2))] = -1
    st["labels"] = st["teacher_index"][:, 0].clone()
    st["labels"][torch.rand(rows, generator=g, device="cuda") < 0.05] = -1
    st["out"] = {"loss": floats(rows)}
    if train:
        st["dloss"] = (0.5 + torch.rand(rows, generator=g, device="cuda")) / rows
        st["out"].update(dlogits=empty(case), stats=floats(rows, 4))
    return st


# ---------------------------------------------------------------------------------------------- one pass
def run(st):
    if own:
        return {"norm": own_norm, "logprob": own_logprob, "distill": own_distill}[st["kind"]](st)
    return {"norm": plain_norm, "logprob": plain_logprob, "distill": plain_distill}[st["kind"]](st)


def own_norm(st):
    from paper_1606_04487_amd import binding as B
    out, x = st["out"], st["x"]
    if st["way"] == "forward":
        y, _, _ = B.layer_norm_forward(x, st["gamma"], st["beta"], EPS, out["y"], want_stats=False)
        return {"y": y}
    y, mean, rstd = B.layer_norm_forward(x, st["gamma"], st["beta"], EPS, out["y"], out["mean"], out["rstd"])
    dx, dgamma, dbeta = B.layer_norm_backward(x, st["dy"], mean, rstd, st["gamma"], out["dx"], out["dgamma"], out["dbeta"])
    return {"y": y, "dx": dx, "dgamma": dgamma, "dbeta": dbeta}


def own_logprob(st):
    from paper_1606_04487_amd import binding as B
    out, x, top, t = st["out"], st["logits"], st["top"], st["temperature"]
    lp, entropy, index, best, stats = B.logprob_forward(x, st["targets"], top, t, logprob=out["logprob"], entropy=out["entropy"],
                                                        top_index=out.get("top_index"), top_logprob=out.get("top_logprob"),
                                                        stats=out["stats"])
    got = {"logprob": lp, "entropy": entropy}
    if top:
        got.update(top_index=index, top_logprob=best)
    if st["way"] == "train":
        got["dlogits"] = B.logprob_backward(x, stats, st["targets"], st["dlogprob"], st["dentropy"], entropy, t, dlogits=out["dlogits"])
    return got


def own_distill(st):
    from paper_1606_04487_amd import binding as B
    out, given = st["out"], (st["logits"], st["teacher_index"], st["teacher_logits"], st["labels"], st["temperature"], st["alpha"])
    if st["way"] == "forward":
        return {"loss": B.distill_forward(*given, loss=out["loss"], want_stats=False)[0]}
    if st["way"] == "both":
        loss, dlogits = B.distill_forward_backward(*given, dloss=st["dloss"], loss=out["loss"], dlogits=out["dlogits"])
        return {"loss": loss, "dlogits": dlogits}
    loss, stats = B.distill_forward(*given, loss=out["loss"], stats=out["stats"])
    return {"loss": loss, "dlogits": B.distill_backward(*given, stats=stats, dloss=st["dloss"], dlogits=out["dlogits"])}


def plain_norm(st):
    x = st["x"].float()
    mean = x.mean(1, keepdim=True)
    centred = x - mean
    rstd = torch.rsqrt((centred * centred).mean(1, keepdim=True) + EPS)
    xhat = centred * rstd
    y = (xhat * st["gamma"] + st["beta"]).to(st["x"].dtype)
    if st["way"] == "forward":
        return {"y": y}
    dy = st["dy"].float()
    g = dy * st["gamma"]
    dx = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    return {"y": y, "dx": dx.to(st["x"].dtype), "dgamma": (dy * xhat).sum(0), "dbeta": dy.sum(0)}


def plain_top(x, k):
    """The k largest of every row, ties to the lowest index: the order of (value, -index) as one 64-bit whole number."""
    bits = x.view(torch.int32)
    order = (bits ^ ((bits >> 31) & 0x7fffffff)).long()       # as the values are ordered
    key = (order << 32) + torch.arange(x.shape[1] - 1, -1, -1, device=x.device)
    best = key.topk(min(k, x.shape[1]), dim=1).values
    index = x.shape[1] - 1 - (best & 0xffffffff)
    value = x.gather(1, index)
    return torch.where(value > -math.inf, index, -1), value


def plain_logprob(st):
    x = st["logits"].float()
    z = (x - x.amax(1, keepdim=True)) / st["temperature"]
    e = z.exp()
    s = e.sum(1, keepdim=True)
    lnsum = s.log()
    p = e / s
    entropy = lnsum - (torch.where(p > 0, z, 0.0) * p).sum(1, keepdim=True)
    at = st["targets"].unsqueeze(1)
    got = {"logprob": (z.gather(1, at) - lnsum).squeeze(1), "entropy": entropy.squeeze(1)}
    if st["top"]:
        got["top_index"], value = plain_top(x, st["top"])
        got["top_logprob"] = (value - x.amax(1, keepdim=True)) / st["temperature"] - lnsum
    if st["way"] == "train":
        dlp, dh = st["dlogprob"].unsqueeze(1), st["dentropy"].unsqueeze(1)
        lp = torch.where(p > 0, z - lnsum, 0.0)
        d = -p * (dlp + dh * (lp + entropy))
        d.scatter_add_(1, at, dlp)
        got["dlogits"] = (d / st["temperature"]).to(st["logits"].dtype)
    return got


def plain_distill(st):
    x, t, alpha = st["logits"].float(), st["temperature"], st["alpha"]
    index, labels = st["teacher_index"], st["labels"].unsqueeze(1)
    live, has = index >= 0, labels >= 0
    at, label = index.clamp(min=0), labels.clamp(min=0)
    tz = torch.where(live, st["teacher_logits"], -math.inf) / t
    tz = tz - tz.amax(1, keepdim=True)
    te = tz.exp()
    q = te / te.sum(1, keepdim=True)
    lnq = torch.where(live, tz - te.sum(1, keepdim=True).log(), 0.0)
    z1 = x - x.amax(1, keepdim=True)
    e1 = z1.exp()
    s1 = e1.sum(1, keepdim=True)
    z = z1 / t
    e = z.exp()
    s = e.sum(1, keepdim=True)
    kl = (q * (lnq - (z.gather(1, at) - s.log()))).sum(1)
    ce = torch.where(has, s1.log() - z1.gather(1, label), 0.0).squeeze(1)
    loss = alpha * t * t * kl + (1.0 - alpha) * ce
    if st["way"] == "forward":
        return {"loss": loss}
    d = (e / s).scatter_add_(1, at, -q) * (alpha * t)
    d += (1.0 - alpha) * has * (e1 / s1).scatter_add_(1, label, torch.full_like(s, -1.0))
    return {"loss": loss, "dlogits": (d * st["dloss"].unsqueeze(1)).to(st["logits"].dtype)}


# ---------------------------------------------------------------------------------------------- what a pass needs
def work(case):
    """Every input read once and every output written once; an exponential counts as one operation."""
    e, rows, width, train = 2 if case["dtype"] == "bf16" else 4, case["rows"], case["width"], case["way"] != "forward"
    n = rows * width
    if case["kind"] == "norm":
        # forward: x in, y out; training also takes dy in and gives dx, the weights' gradients and the rows' statistics
        return {"bytes": (4 if train else 2) * n * e + (16 if train else 8) * width + (8 * rows if train else 0), "flops": (22 if train else 8) * n}
    if case["kind"] == "logprob":
        small = rows * (8 + 4 + 4 + 8 + 12 * case["top"] + (8 if train else 0))
        return {"bytes": (2 if train else 1) * n * e + small, "flops": (14 if train else 6) * n}
    small = rows * (12 * case["kept"] + 8 + 4 + (4 if train else 0))
    exps = 1 if case["alpha"] == 1.0 or case["temperature"] == 1.0 else 2
    return {"bytes": (2 if train else 1) * n * e + small, "flops": (9 if train else 4) * exps * n}


# ---------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    """What `run` gives for these inputs, from the definitions in 64 bits, a few rows at a time."""
    st = prepare(case, seed)
    at = {"norm": "x", "logprob": "logits", "distill": "logits"}[case["kind"]]
    step = max(1, (1 << 26) // case["width"])
    parts = []
    for lo in range(0, case["rows"], step):
        rows = slice(lo, lo + step)
        part = {k: v[rows].double() if v.is_floating_point() else v[rows] for k, v in st.items()
                if torch.is_tensor(v) and k not in ("gamma", "beta")}
        parts.append({"norm": exact_norm, "logprob": exact_logprob, "distill": exact_distill}[case["kind"]](part[at], part, st))
    whole = {k: sum(p[k] for p in parts) if k in ("dgamma", "dbeta") else torch.cat([p[k] for p in parts]) for k in parts[0]}
    if "top_logprob" in whole:  # the indices are held to equality as they are
        return {k: v for k, v in [("logprob", whole["logprob"]), ("entropy", whole["entropy"]), ("top_index", None),
                                  ("top_logprob", whole["top_logprob"]), ("dlogits", whole.get("dlogits"))] if k != "dlogits" or v is not None}
    return whole


def exact_norm(x, part, st):
    var, mean = torch.var_mean(x, dim=1, unbiased=False, keepdim=True)
    xhat = (x - mean) / (var + EPS).sqrt()
    gamma = st["gamma"].double()
    got = {"y": xhat * gamma + st["beta"].double()}
    if st["way"] == "train":
        dy, n = part["dy"], x.shape[1]
        dxhat = dy * gamma
        got["dx"] = (n * dxhat - dxhat.sum(1, keepdim=True) - xhat * (dxhat * xhat).sum(1, keepdim=True)) / (n * (var + EPS).sqrt())
        got["dgamma"], got["dbeta"] = (dy * xhat).sum(0), dy.sum(0)
    return got


def exact_logprob(x, part, st):
    lp = torch.log_softmax(x / st["temperature"], dim=1)
    p = lp.exp()
    plogp = torch.special.entr(p)
    got = {"logprob": lp.gather(1, part["targets"][:, None])[:, 0], "entropy": plogp.sum(1)}
    if st["top"]:
        got["top_logprob"] = lp.topk(st["top"], dim=1).values
    if st["way"] == "train":
        # d entropy / dz = entr(p) - p H, d lp_t / dz = onehot - p
        d = part["dentropy"][:, None] * (plogp - p * got["entropy"][:, None]) - part["dlogprob"][:, None] * p
        r = torch.arange(x.shape[0], device=x.device)
        d[r, part["targets"]] += part["dlogprob"]
        got["dlogits"] = d / st["temperature"]
    return got


def exact_distill(x, part, st):
    t, alpha, index, labels = st["temperature"], st["alpha"], part["teacher_index"], part["labels"]
    r = torch.arange(x.shape[0], device=x.device)
    lnq = torch.log_softmax(part["teacher_logits"].masked_fill(index < 0, -math.inf) / t, dim=1)
    q = torch.zeros_like(x)
    q.scatter_(1, index.clamp(min=0), 0.0)
    row, col = (index >= 0).nonzero(as_tuple=True)
    q[row, index[row, col]] = lnq[row, col].exp()
    lp, lp1 = torch.log_softmax(x / t, dim=1), torch.log_softmax(x, dim=1)
    kl = (torch.xlogy(q, q) - q * lp).sum(1)
    has = (labels >= 0).double()
    ce = -lp1[r, labels.clamp(min=0)] * has
    got = {"loss": alpha * t * t * kl + (1 - alpha) * ce}
    if st["way"] != "forward":
        hard = lp1.exp()
        hard[r, labels.clamp(min=0)] -= 1.0
        got["dlogits"] = part["dloss"][:, None] * (alpha * t * (lp.exp() - q) + (1 - alpha) * has[:, None] * hard)
    return got
