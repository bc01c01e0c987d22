"""Timing cases of the operators at the two ends of a training step around the blocks: the scaled lookup
of token embeddings and its gradient, the cross-entropy of a vocabulary with its gradient, and the
orthogonalised update that a weight's accumulated gradient becomes.

``run`` computes them in elementary torch operations where ``own`` is false and through the entry points
of ``paper_2605_25451_amd.binding`` where it is true.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
CODES = {"bf16": 0, "fp32": 1}                       # BM_DTYPE_*
COEFFICIENTS = (3.4445, -4.7750, 2.0315)             # of the quintic Newton-Schulz iteration
STEPS, EPS = 5, 1e-7


# ---- the cases -----------------------------------------------------------------------------------

def listed():
    return [
        # one token: what a call costs
        {"name": "embed_1", "kind": "embed", "type": "bf16", "tokens": 1, "vocab": 32000, "width": 4096, "images": 0.0},
        # a microbatch of interleaved image and text spans: the rows of image tokens are left alone
        {"name": "embed_8192", "kind": "embed", "type": "bf16", "tokens": 8192, "vocab": 128000, "width": 4096, "images": 0.45},
        # the gradient of one short document of odd length
        {"name": "embed_grad_777", "kind": "embed_grad", "type": "bf16", "tokens": 777, "vocab": 32000, "width": 4096, "images": 0.0},
        # the fp32 path: a small model's odd vocabulary
        {"name": "embed_grad_fp32_5000", "kind": "embed_grad", "type": "fp32", "tokens": 5000, "vocab": 50257, "width": 768, "images": 0.1},
        # a long pack; the words of a language are drawn by their rank, so few rows take many tokens
        {"name": "embed_grad_32768", "kind": "embed_grad", "type": "bf16", "tokens": 32768, "vocab": 64000, "width": 4096, "images": 0.0},
        # the last few rows of a pack, answers only: most labels are ignored
        {"name": "loss_48", "kind": "loss", "type": "bf16", "tokens": 48, "vocab": 32000, "ignored": 0.7},
        # an odd vocabulary: rows that start off every boundary
        {"name": "loss_fp32_1000", "kind": "loss", "type": "fp32", "tokens": 1000, "vocab": 50257, "ignored": 0.1},
        # half a microbatch on a large vocabulary
        {"name": "loss_4096", "kind": "loss", "type": "bf16", "tokens": 4096, "vocab": 128000, "ignored": 0.3},
        # a small block's matrix, taller than wide: latency and launches
        {"name": "ortho_192x64", "kind": "ortho", "type": "bf16", "batch": 1, "rows": 192, "cols": 64},
        # the output projection of a generator block on the fp32 path
        {"name": "ortho_fp32_1152x1152", "kind": "ortho", "type": "fp32", "batch": 1, "rows": 1152, "cols": 1152},
        # the down projection of a large decoder block
        {"name": "ortho_4096x14336", "kind": "ortho", "type": "bf16", "batch": 1, "rows": 4096, "cols": 14336},
        # the up projections of a block's 128 experts
        {"name": "ortho_128_1536x2048", "kind": "ortho", "type": "bf16", "batch": 128, "rows": 1536, "cols": 2048},
    ]


def _log(rng, lo, hi):
    """An integer of [lo, hi], uniform in its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["embed", "embed_grad", "embed_grad", "loss", "loss", "ortho", "ortho", "ortho"])
    kind_type = rng.choice(["bf16", "bf16", "fp32"])
    case = {"kind": kind, "type": kind_type}
    if kind in ("embed", "embed_grad"):
        case["tokens"] = _log(rng, 1, 32768)
        case["vocab"] = _log(rng, 1000, 64000)
        case["width"] = 8 * _log(rng, 8, 512)
        case["images"] = round(rng.choice([0.0, rng.uniform(0.0, 0.6)]), 3)
    elif kind == "loss":
        case["vocab"] = _log(rng, 300, 128000)
        case["tokens"] = _log(rng, 1, max(1, min(8192, (1 << (29 if kind_type == "bf16" else 28)) // case["vocab"])))
        case["ignored"] = round(rng.uniform(0.0, 0.8), 3)
    else:
        case["batch"] = rng.choice([1, 1, _log(rng, 1, 64)])
        most = 4096 if case["batch"] == 1 else 1024
        case["rows"], case["cols"] = _log(rng, 16, most), _log(rng, 16, most)
    return case


# ---- inputs ----------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _words(case, g):
    """Token ids by rank (the k-th most frequent word as often as 1/k), ranks shuffled over the ids; -1 on image rows."""
    u = torch.rand(case["tokens"], device=DEVICE, generator=g, dtype=torch.float64)
    rank = (torch.exp(u * math.log(case["vocab"] + 1)) - 1).long().clamp_(0, case["vocab"] - 1)
    ids = torch.randperm(case["vocab"], device=DEVICE, generator=g)[rank].int()
    if case["images"]:
        ids[torch.rand(case["tokens"], device=DEVICE, generator=g) < case["images"]] = -1
    return ids


def _normal(shape, g, type_=torch.float32, std=1.0):
    return (torch.randn(shape, device=DEVICE, generator=g) * std).to(type_)


def inputs(case, seed):
    g = _generator(seed)
    kind, type_ = case["kind"], TYPES[case["type"]]
    if kind == "embed":
        return {"ids": _words(case, g), "table": _normal((case["vocab"], case["width"]), g, type_, 0.02),
                "y": _normal((case["tokens"], case["width"]), g, type_)}
    if kind == "embed_grad":
        return {"ids": _words(case, g), "dy": _normal((case["tokens"], case["width"]), g, type_, 0.1),
                "dtable": _normal((case["vocab"], case["width"]), g, torch.float32, 0.01)}
    if kind == "loss":
        T, V = case["tokens"], case["vocab"]
        logits = _normal((T, V), g, type_, 2.0)
        labels = torch.randint(0, V, (T,), device=DEVICE, generator=g, dtype=torch.int32)
        rows = torch.arange(T, device=DEVICE)
        logits[rows, labels.long()] += (6 * torch.rand(T, device=DEVICE, generator=g)).to(type_)     # a model that has learnt something
        labels[torch.rand(T, device=DEVICE, generator=g) < case["ignored"]] = -1
        return {"logits": logits, "labels": labels, "weight": torch.rand(T, device=DEVICE, generator=g) / T}
    # a gradient: a few strong directions that decay, over noise
    B, M, N = case["batch"], case["rows"], case["cols"]
    rank = max(1, min(M, N) // 8)
    grad = _normal((B, M, N), g, std=1e-3)
    decay = torch.arange(1, rank + 1, device=DEVICE, dtype=torch.float32).pow_(-0.7)
    grad += torch.matmul(_normal((B, M, rank), g, std=0.05) * decay, _normal((B, rank, N), g, std=0.1))
    return {"grad": grad}


def prepare(case, seed):
    s = dict(inputs(case, seed), case=case, type=TYPES[case["type"]], code=CODES[case["type"]])
    kind = case["kind"]
    if kind in ("embed", "embed_grad"):
        s["scale"] = math.sqrt(case["width"])
    if kind == "loss":
        s["loss"] = torch.zeros(case["tokens"], device=DEVICE)
        s["dlogits"] = torch.zeros_like(s["logits"])
    if kind == "ortho":
        s["update"] = torch.zeros(s["grad"].shape, device=DEVICE, dtype=s["type"])
    if own:
        from paper_2605_25451_amd import binding as bm
        n = 0
        if kind == "embed_grad":
            n = bm.embedding_backward_scratch_bytes(case["tokens"], case["width"])
        if kind == "loss":
            n = bm.cross_entropy_scratch_bytes(s["code"], case["tokens"], case["vocab"])
        if kind == "ortho":
            n = bm.orthogonalize_scratch_bytes(s["code"], case["batch"], case["rows"], case["cols"])
        s["scratch_bytes"] = n
        s["scratch"] = torch.empty(max(n, 16), dtype=torch.uint8, device=DEVICE)
    return s


# ---- one pass --------------------------------------------------------------------------------------

def _embed(s):
    ids = s["ids"].long()
    rows = s["table"][ids.clamp(min=0)].float() * s["scale"]
    s["y"].copy_(torch.where((ids >= 0)[:, None], rows, s["y"].float()))
    return s["y"]


def _embed_grad(s):
    ids = s["ids"].long()
    rows = s["dy"].float() * s["scale"] * (ids >= 0)[:, None]
    s["dtable"].index_add_(0, ids.clamp(min=0), rows)
    return s["dtable"]


def _loss(s):
    x, labels, weight = s["logits"].float(), s["labels"].long(), s["weight"]
    weight = torch.where(labels >= 0, weight, torch.zeros_like(weight))
    labels = labels.clamp(min=0)[:, None]
    top = x.amax(dim=1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(dim=1, keepdim=True)
    loss = weight * (top + torch.log(total) - x.gather(1, labels))[:, 0]
    p = e / total
    p.scatter_add_(1, labels, torch.full_like(total, -1.0))
    return {"loss": loss, "dlogits": (p * weight[:, None]).to(s["type"])}


def _newton_schulz(s):
    a, b, c = COEFFICIENTS
    x = s["grad"]
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2).contiguous()
    x = x / (torch.sqrt((x.double() * x.double()).sum(dim=(1, 2), keepdim=True)) + EPS).float()
    for _ in range(STEPS):
        gram = torch.matmul(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.matmul(b * gram + c * torch.matmul(gram, gram), x)
    return (x.transpose(1, 2) if tall else x).to(s["type"]).contiguous()


def run(state):
    s, case = state, state["case"]
    kind = case["kind"]
    if own:
        from paper_2605_25451_amd import binding as bm
        if kind == "embed":
            bm.embedding_forward(s["code"], case["vocab"], case["width"], s["table"], case["width"], s["ids"], case["tokens"],
                                 s["scale"], s["y"], case["width"])
            return s["y"]
        if kind == "embed_grad":
            bm.embedding_backward(s["code"], case["vocab"], case["width"], s["dy"], case["width"], s["ids"], case["tokens"],
                                  s["scale"], s["dtable"], case["width"], s["scratch"], s["scratch_bytes"])
            return s["dtable"]
        if kind == "loss":
            bm.cross_entropy(s["code"], case["tokens"], case["vocab"], s["logits"], case["vocab"], s["labels"], s["weight"],
                             s["loss"], s["dlogits"], case["vocab"], s["scratch"], s["scratch_bytes"])
            return {"loss": s["loss"], "dlogits": s["dlogits"]}
        M, N = case["rows"], case["cols"]
        bm.orthogonalize(s["code"], case["batch"], M, N, s["grad"], N, M * N, s["update"], N, M * N, COEFFICIENTS, STEPS, EPS,
                         s["scratch"], s["scratch_bytes"])
        return s["update"]
    if kind == "embed":
        return _embed(s)
    if kind == "embed_grad":
        return _embed_grad(s)
    return _loss(s) if kind == "loss" else _newton_schulz(s)


# ---- what a pass cannot do without -------------------------------------------------------------------

def _distinct(case):
    """Expected number of different words among the text tokens."""
    n, V = case["tokens"] * (1 - case["images"]), case["vocab"]
    total, k, lo = 0.0, math.log(V + 1), 1
    while lo <= V:                                    # over runs of ranks that double
        hi = min(V, 2 * lo - 1)
        p = math.log((hi + 1) / lo) / k / (hi - lo + 1)
        total += (hi - lo + 1) * -math.expm1(n * math.log1p(-min(p, 1 - 1e-12)))
        lo = hi + 1
    return max(1.0, total)


def work(case):
    size = 2 if case["type"] == "bf16" else 4
    kind = case["kind"]
    if kind in ("embed", "embed_grad"):
        T, d = case["tokens"], case["width"]
        text, words = T * (1 - case["images"]), _distinct(case)
        if kind == "embed":
            return {"bytes": 4 * T + (words + text) * d * size, "flops": text * d}
        return {"bytes": 4 * T + text * d * size + 2 * words * d * 4, "flops": 2 * text * d}
    if kind == "loss":
        # a row whose label is ignored is not read, but its gradient is written
        T, V = case["tokens"], case["vocab"]
        return {"bytes": T * (V * size * (2 - case["ignored"]) + 12), "flops": 5.0 * T * V * (1 - case["ignored"])}
    B, M, N = case["batch"], case["rows"], case["cols"]
    m, n = min(M, N), max(M, N)
    # the two symmetric products need one triangle
    return {"bytes": B * M * N * (4 + size), "flops": STEPS * B * (float(m) * m * n + float(m) ** 3 + 2.0 * m * m * n)}


# ---- the definitions in 64 bits ----------------------------------------------------------------------

def exact(case, seed):
    x = inputs(case, seed)
    kind = case["kind"]
    if kind == "embed":
        y, ids = x["y"].double(), x["ids"].long()
        text = torch.nonzero(ids >= 0)[:, 0]
        y[text] = math.sqrt(case["width"]) * torch.index_select(x["table"], 0, ids[text]).double()
        return y
    if kind == "embed_grad":
        ids = x["ids"].long()
        text = torch.nonzero(ids >= 0)[:, 0]
        out = x["dtable"].double()
        rows = x["dy"][text].double() * math.sqrt(case["width"])
        return out.index_put_((ids[text],), rows, accumulate=True)
    if kind == "loss":
        labels = x["labels"].long()
        loss = torch.zeros(case["tokens"], device=DEVICE, dtype=torch.float64)
        grad = torch.zeros(x["logits"].shape, device=DEVICE, dtype=torch.float64)
        live = torch.nonzero(labels >= 0)[:, 0]
        for part in torch.split(live, 512):
            z = x["logits"][part].double()
            w = x["weight"][part].double()
            lse = torch.logsumexp(z, dim=1)
            here = torch.arange(len(part), device=DEVICE)
            loss[part] = w * (lse - z[here, labels[part]])
            p = torch.exp(z - lse[:, None])
            p[here, labels[part]] -= 1.0
            grad[part] = w[:, None] * p
        return {"loss": loss, "dlogits": grad}
    a, b, c = COEFFICIENTS
    out = torch.empty(x["grad"].shape, device=DEVICE, dtype=torch.float64)
    for i in range(case["batch"]):
        y = x["grad"][i].double()
        wide = y.shape[0] < y.shape[1]
        y = y.t().contiguous() if wide else y
        y = y / (torch.linalg.vector_norm(y) + EPS)
        eye = torch.eye(y.shape[1], device=DEVICE, dtype=torch.float64)
        for _ in range(STEPS):
            s = y.t().contiguous() @ y
            y = y @ (a * eye + s @ (b * eye + c * s))
        out[i] = y.t() if wide else y
    return out
