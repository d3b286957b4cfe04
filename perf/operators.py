"""The calls of a training step around the GNN layer, as a user's program makes them: the embedding lookup with its
gradient, the Update grouped by expert (or node type) with its gradients, and the loss against a teacher's top logits
with the gradient of the student's logits.

Everything is drawn on the GPU from the seed; ids, group offsets and teacher entries are device tensors that change from
step to step.  A program keeps its weights, tables and workspaces, and its outputs come from torch's allocator.
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda"
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


def _binding():
    from paper_2209_06800_amd import binding
    return binding


# ---- the cases -----------------------------------------------------------------------------------------------
def listed():
    return [
        # One token looked up at a serving step: latency alone.
        dict(name="lookup_1_of_32k_dim4096", kind="embed", n=1, rows=32000, dim=4096, table="bf16", out="bf16", ids="i64", scale=64.0),
        # A long batch of tokens at training, wide rows scaled on the way out.
        dict(name="lookup_64k_of_128k_dim2048", kind="embed", n=65536, rows=128000, dim=2048, table="bf16", out="bf16", ids="i64", scale=45.25),
        # Gradient of a small table from a short batch, fp32, an odd width; padding tokens carry none.
        dict(name="lookup_grad_2k_of_5k_dim602", kind="embed_grad", n=2049, rows=5003, dim=602, grad="f32", out="f32", ids="i32", scale=1.0, accumulate=False),
        # Gradient of a large table from a long batch of skewed tokens (the commonest one some 8 % of them).
        dict(name="lookup_grad_32k_of_128k_dim2048", kind="embed_grad", n=32768, rows=128000, dim=2048, grad="bf16", out="f32", ids="i64", scale=45.25,
             accumulate=False),
        # A serving step: 64 rows over 64 experts, most of the time goes into reading weights.
        dict(name="grouped_64_of_64x1024to2048", kind="grouped", n=64, groups=64, d_in=1024, d_out=2048, dtype="bf16", out="bf16", act="none", bias=False, skew=0.7),
        # Node types of a heterogeneous graph, one linear each, fp32, widths of a product graph's first layer.
        dict(name="grouped_233k_of_7x100to256_f32", kind="grouped", n=232965, groups=7, d_in=100, d_out=256, dtype="f32", out="f32", act="relu", bias=True, skew=1.0),
        # The first product of the experts at training, ragged shares of a long batch.
        dict(name="grouped_32k_of_8x4096to4096", kind="grouped", n=32768, groups=8, d_in=4096, d_out=4096, dtype="bf16", out="bf16", act="relu", bias=True, skew=0.5),
        # Gradients of a small fp32 layer with odd widths (602 features, 47 classes) and a type that has no node.
        dict(name="grouped_grad_5k_of_5x602to47_f32", kind="grouped_grad", n=5003, groups=5, d_in=602, d_out=47, dtype="f32", dw="f32", act="none", bias=True,
             skew=1.0, accumulate=False),
        # Gradients of the experts' first product: rows, weights and biases, through the ReLU.
        dict(name="grouped_grad_16k_of_8x2048to4096", kind="grouped_grad", n=16384, groups=8, d_in=2048, d_out=4096, dtype="bf16", dw="f32", act="relu", bias=True,
             skew=0.5, accumulate=False),
        # A GNN distilled into another over 47 classes: the loss of all nodes, no gradient wanted.
        dict(name="distill_306k_of_47_top8_f32", kind="distill", n=306128, classes=47, k=8, logits="f32", top="f32", ids="i32", temperature=2.0, grad="none",
             masked=0.1),
        # One short sequence against a large vocabulary, with the gradient.
        dict(name="distill_grad_37_of_50k_top20", kind="distill", n=37, classes=50021, k=20, logits="bf16", top="f32", ids="i64", temperature=1.0, grad="bf16",
             masked=0.2),
        # A training batch of tokens, a large vocabulary, 64 teacher entries each.
        dict(name="distill_grad_4k_of_128k_top64", kind="distill", n=4096, classes=128000, k=64, logits="bf16", top="bf16", ids="i64", temperature=2.0, grad="bf16",
             masked=0.1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Half of them the multiples of 64 that people choose, half whatever comes."""
    w = _log(rng, lo, hi)
    return w if rng.random() < 0.5 else max(64, w // 64 * 64)


def draw(rng):
    kind = rng.choice(["embed", "embed_grad", "grouped", "grouped", "grouped_grad", "grouped_grad", "distill", "distill"])
    if kind == "embed":
        dim = _width(rng, 16, 5000)
        return dict(kind=kind, n=_log(rng, 1, min(1 << 20, (1 << 27) // dim)), rows=_log(rng, 300, min(1 << 20, (1 << 28) // dim)), dim=dim,
                    table=rng.choice(["f32", "bf16"]), out=rng.choice(["f32", "bf16"]), ids=rng.choice(["i32", "i64"]), scale=rng.choice([1.0, math.sqrt(dim)]))
    if kind == "embed_grad":
        dim = _width(rng, 16, 5000)
        return dict(kind=kind, n=_log(rng, 1, min(1 << 20, (1 << 26) // dim)), rows=_log(rng, 300, min(1 << 20, (1 << 28) // dim)), dim=dim,
                    grad=rng.choice(["f32", "bf16"]), out=rng.choice(["f32", "f32", "bf16"]), ids=rng.choice(["i32", "i64"]),
                    scale=rng.choice([1.0, math.sqrt(dim)]), accumulate=rng.random() < 0.3)
    if kind in ("grouped", "grouped_grad"):
        dtype = rng.choice(["bf16", "bf16", "f32"])
        groups, d_in, d_out = _log(rng, 1, 128), _width(rng, 16, 4096), _width(rng, 16, 4096)
        groups = max(1, min(groups, (1 << 28) // (d_in * d_out)))
        most = (1 << 38 if kind == "grouped" else 1 << 36) // (d_in * d_out) // (1 if dtype == "bf16" else 4)
        c = dict(kind=kind, n=_log(rng, 1, max(2, min(most, 1 << 18))), groups=groups, d_in=d_in, d_out=d_out, dtype=dtype, act=rng.choice(["none", "relu"]),
                 bias=rng.random() < 0.5, skew=rng.choice([0.0, 0.5, 1.0, 2.0]))
        if kind == "grouped":
            c["out"] = "f32" if dtype == "f32" else rng.choice(["bf16", "bf16", "f32"])
        else:
            c.update(dw="f32" if dtype == "f32" else rng.choice(["f32", "bf16"]), accumulate=rng.random() < 0.3)
        return c
    classes = _log(rng, 5, 260000)
    logits = rng.choice(["f32", "bf16", "bf16"])
    return dict(kind=kind, n=_log(rng, 1, min(400000, (1 << 28) // classes)), classes=classes, k=min(_log(rng, 1, 128), max(1, classes // 3)), logits=logits,
                top=rng.choice(["f32", "bf16"]), ids=rng.choice(["i32", "i64"]), temperature=rng.choice([1.0, 2.0, 4.0, rng.uniform(0.5, 5.0)]),
                grad=rng.choice(["none", logits, logits]), masked=rng.choice([0.0, 0.1, 0.4]))


# ---- inputs --------------------------------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _normal(g, *shape, dtype="f32", std=1.0):
    t = torch.randn(*shape, device=DEV, generator=g, dtype=DTYPE[dtype])
    return t if std == 1.0 else t.mul_(std)


def _ids(case, g):
    """Token ids by a truncated power law (exponent 1), ranks spread over the table; one in 16 is padding (-1) in a longer batch."""
    n, rows = case["n"], case["rows"]
    rank = torch.exp(torch.rand(n, device=DEV, generator=g, dtype=torch.float64) * math.log(rows + 1.0)).floor_().long().sub_(1).clamp_(0, rows - 1)
    step = int(rows * 0.6180339887) | 1
    while math.gcd(step, rows) != 1:
        step += 2
    ids = (rank * step + 17) % rows
    if n >= 16:
        ids = torch.where(torch.rand(n, device=DEV, generator=g) < 1 / 16, -1, ids)
    return ids if case["ids"] == "i64" else ids.int()


def _group_ptr(case, seed):
    rng = np.random.default_rng([int(seed), 71])
    p = np.exp(case["skew"] * rng.standard_normal(case["groups"]))
    if case["groups"] >= 5:
        p[int(rng.integers(case["groups"]))] = 0.0         # one that no row is sent to
    count = rng.multinomial(case["n"], p / p.sum())
    return np.concatenate([[0], np.cumsum(count)]).astype(np.int64)


def prepare(case, seed):
    g, kind = _generator(seed), case["kind"]
    s = dict(case=case)
    if kind == "embed":
        s["ids"], s["table"] = _ids(case, g), _normal(g, case["rows"], case["dim"], dtype=case["table"], std=0.02)
        return s
    if kind == "embed_grad":
        s["ids"], s["grad"] = _ids(case, g), _normal(g, case["n"], case["dim"], dtype=case["grad"], std=1e-3)
        if case["accumulate"]:          # the gradient of an earlier micro-batch
            s["into"] = _normal(g, case["rows"], case["dim"], dtype=case["out"], std=1e-3)
        if own:
            s["workspace"] = torch.empty(_binding().mgg_embed_grad_workspace_bytes(case["n"], case["rows"], case["dim"]), dtype=torch.uint8, device=DEV)
        return s
    if kind in ("grouped", "grouped_grad"):
        d_in, d_out, dt = case["d_in"], case["d_out"], case["dtype"]
        ptr = _group_ptr(case, seed)
        s["ptr"] = torch.from_numpy(ptr).to(DEV)
        s["a"] = _normal(g, case["n"], d_in, dtype=dt)
        s["w"] = _normal(g, case["groups"], d_in, d_out, dtype=dt, std=d_in ** -0.5)
        s["bias"] = _normal(g, case["groups"], d_out, std=0.1) if case["bias"] else None
        if kind == "grouped":
            return s
        s["grad"] = _normal(g, case["n"], d_out, dtype=dt, std=1e-2)
        if case["act"] == "relu":       # what the forward pass left
            s["out"] = torch.empty(case["n"], d_out, dtype=DTYPE[dt], device=DEV)
            for e in range(case["groups"]):
                rows = slice(int(ptr[e]), int(ptr[e + 1]))
                s["out"][rows] = torch.relu(s["a"][rows] @ s["w"][e])
        if case["accumulate"]:
            s["into"] = _normal(g, case["groups"], d_in, d_out, dtype=case["dw"], std=1e-2)
        if own:
            need = _binding().mgg_update_grouped_grad_workspace_bytes(case["n"], case["groups"], d_in, d_out, s["a"].dtype, act=case["act"])
            s["workspace"] = torch.empty(need, dtype=torch.uint8, device=DEV)
        return s
    n, classes, k = case["n"], case["classes"], case["k"]
    logits = _normal(g, n, classes, dtype=case["logits"], std=2.0)
    # distinct classes of each row: a stride from a random one; the teacher's logits fall off from the first
    stride = torch.randint(1, max(2, classes // k), (n, 1), device=DEV, generator=g)
    ids = (torch.randint(0, classes, (n, 1), device=DEV, generator=g) + stride * torch.arange(k, device=DEV)) % classes
    top = (math.log(classes) + 1.0 - torch.arange(k, device=DEV) * (6.0 / k) + _normal(g, n, k)).to(DTYPE[case["top"]])
    logits.scatter_add_(1, ids, (top.float() * torch.rand(n, 1, device=DEV, generator=g)).to(logits.dtype))     # a student on its way there
    if k > 4:                           # some teachers kept fewer entries
        ids = torch.where(torch.rand(n, k, device=DEV, generator=g) < 0.05, -1, ids)
    keep = torch.rand(n, device=DEV, generator=g) >= case["masked"]
    s.update(logits=logits, ids=ids if case["ids"] == "i64" else ids.int(), top=top, weight=keep.float() / n)
    if own:
        s["workspace"] = torch.empty(_binding().mgg_distill_workspace_bytes(n, classes), dtype=torch.uint8, device=DEV)
    return s


# ---- one pass ------------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    return (_run_own if own else _run_plain)[case["kind"]](s, case)


def _own_embed(s, case):
    return _binding().mgg_embed(s["ids"], s["table"], scale=case["scale"], out_dtype=DTYPE[case["out"]])


def _own_embed_grad(s, case):
    out = s["into"].clone() if case["accumulate"] else None
    return _binding().mgg_embed_grad(s["ids"], s["grad"], case["rows"], scale=case["scale"], out=out, out_dtype=DTYPE[case["out"]],
                                     accumulate=case["accumulate"], workspace=s["workspace"])


def _own_grouped(s, case):
    return _binding().mgg_update_grouped(s["ptr"], s["a"], s["w"], s["bias"], case["act"], out_dtype=DTYPE[case["out"]])


def _own_grouped_grad(s, case):
    grad_w = s["into"].clone() if case["accumulate"] else None
    return _binding().mgg_update_grouped_grad(s["ptr"], s["grad"], s["a"], s["w"], case["act"], out=s.get("out"), grad_w=grad_w, w_grad_dtype=DTYPE[case["dw"]],
                                              need_bias=case["bias"], accumulate=case["accumulate"], workspace=s["workspace"])


def _own_distill(s, case):
    return _binding().mgg_distill_loss(s["logits"], s["ids"], s["top"], temperature=case["temperature"], row_weight=s["weight"],
                                       need_grad=case["grad"] != "none", workspace=s["workspace"])


def _plain_embed(s, case):
    ids = s["ids"].long()
    rows = s["table"].index_select(0, ids.clamp_min(0)).float() * case["scale"]
    return torch.where((ids >= 0)[:, None], rows, 0.0).to(DTYPE[case["out"]])


def _plain_embed_grad(s, case):
    ids = s["ids"].long()
    total = torch.zeros(case["rows"], case["dim"], device=DEV)
    grad = torch.where((ids >= 0)[:, None], s["grad"].float(), 0.0)
    total.index_add_(0, ids.clamp_min(0), grad)
    total = total * case["scale"]
    if case["accumulate"]:
        total = total + s["into"].float()
    return total.to(DTYPE[case["out"]])


def _plain_grouped(s, case):
    ptr = s["ptr"].tolist()
    out = torch.empty(case["n"], case["d_out"], dtype=DTYPE[case["out"]], device=DEV)
    for e in range(case["groups"]):
        rows = slice(ptr[e], ptr[e + 1])
        if ptr[e] == ptr[e + 1]:
            continue
        z = s["a"][rows].float() @ s["w"][e].float()
        if case["bias"]:
            z = z + s["bias"][e]
        out[rows] = (torch.relu(z) if case["act"] == "relu" else z).to(out.dtype)
    return out


def _plain_grouped_grad(s, case):
    ptr = s["ptr"].tolist()
    grad_a = torch.empty_like(s["a"])
    grad_w = torch.zeros(case["groups"], case["d_in"], case["d_out"], dtype=DTYPE[case["dw"]], device=DEV)
    grad_bias = torch.zeros(case["groups"], case["d_out"], device=DEV)
    for e in range(case["groups"]):
        rows = slice(ptr[e], ptr[e + 1])
        dz = s["grad"][rows].float()
        if case["act"] == "relu":
            dz = dz * (s["out"][rows] > 0)
        grad_a[rows] = (dz @ s["w"][e].float().t()).to(grad_a.dtype)
        product = s["a"][rows].float().t() @ dz
        grad_w[e] = (product + s["into"][e].float() if case["accumulate"] else product).to(grad_w.dtype)
        grad_bias[e] = dz.sum(0)
    return (grad_a, grad_w, grad_bias) if case["bias"] else (grad_a, grad_w)


def _plain_distill(s, case):
    t = case["temperature"]
    z = s["logits"].float() / t
    present = s["ids"] >= 0
    ids = s["ids"].long().clamp_min(0)
    teacher = torch.where(present, s["top"].float() / t, -math.inf)
    high = teacher.max(1, keepdim=True).values
    some = torch.isfinite(high)
    p = torch.exp(teacher - torch.where(some, high, 0.0))
    p = p / torch.where(some, p.sum(1, keepdim=True), 1.0)
    log_p = torch.log(torch.where(p > 0, p, 1.0))
    z = z - z.max(1, keepdim=True).values
    e = torch.exp(z)
    total = e.sum(1, keepdim=True)
    log_q = z.gather(1, ids) - torch.log(total)
    w = torch.where(some[:, 0], s["weight"], 0.0)
    loss = w * t * t * torch.where(p > 0, p * (log_p - log_q), 0.0).sum(1)
    if case["grad"] == "none":
        return loss
    dz = (e / total).scatter_add_(1, ids, -p) * (w * t)[:, None]
    return loss, dz.to(DTYPE[case["grad"]])


_run_own = dict(embed=_own_embed, embed_grad=_own_embed_grad, grouped=_own_grouped, grouped_grad=_own_grouped_grad, distill=_own_distill)
_run_plain = dict(embed=_plain_embed, embed_grad=_plain_embed_grad, grouped=_plain_grouped, grouped_grad=_plain_grouped_grad, distill=_plain_distill)


# ---- the definition in 64 bits -------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "embed":
        padded = torch.cat([s["table"].double() * case["scale"], torch.zeros(1, case["dim"], device=DEV, dtype=torch.float64)])
        return padded[s["ids"].long()]             # -1 is the row of zeros at the end
    if kind == "embed_grad":
        order = torch.argsort(s["ids"].long(), stable=True)
        order = order[s["ids"].long()[order] >= 0]
        which, count = torch.unique_consecutive(s["ids"].long()[order], return_counts=True)
        out = s["into"].double() if case["accumulate"] else torch.zeros(case["rows"], case["dim"], device=DEV, dtype=torch.float64)
        if order.numel():
            end = count.cumsum(0)
            width = max(1, (1 << 27) // order.numel())
            for c in range(0, case["dim"], width):      # sums of runs of equal ids as differences of the running sum
                run_sum = torch.cat([torch.zeros(1, min(width, case["dim"] - c), device=DEV, dtype=torch.float64),
                                     s["grad"][order, c:c + width].double().cumsum(0)])
                out[which, c:c + width] += case["scale"] * (run_sum[end] - run_sum[end - count])
        return out
    if kind in ("grouped", "grouped_grad"):
        if 2.0 * case["n"] * case["d_in"] * case["d_out"] > 2e12:
            return None
        group = torch.bucketize(torch.arange(case["n"], device=DEV), s["ptr"][1:], right=True)
        present = [e for e in range(case["groups"]) if bool((group == e).any())]
        if kind == "grouped":
            out = torch.empty(case["n"], case["d_out"], device=DEV, dtype=torch.float64)
            for e in present:
                at = torch.nonzero(group == e)[:, 0]
                out[at] = torch.mm(s["a"][at].double(), s["w"][e].double())
            if case["bias"]:
                out += s["bias"].double()[group]
            return out.clamp_min(0.0) if case["act"] == "relu" else out
        dz = s["grad"].double()
        if case["act"] == "relu":
            dz = torch.where(s["out"] > 0, dz, 0.0)
        grad_a = torch.empty(case["n"], case["d_in"], device=DEV, dtype=torch.float64)
        grad_w = s["into"].double() if case["accumulate"] else torch.zeros(case["groups"], case["d_in"], case["d_out"], device=DEV, dtype=torch.float64)
        grad_bias = torch.zeros(case["groups"], case["d_out"], device=DEV, dtype=torch.float64)
        for e in present:
            at = torch.nonzero(group == e)[:, 0]
            grad_a[at] = torch.mm(dz[at], s["w"][e].double().t().contiguous())
            grad_w[e] += torch.mm(s["a"][at].double().t().contiguous(), dz[at])
            grad_bias[e] = dz[at].sum(0)
        return (grad_a, grad_w, grad_bias) if case["bias"] else (grad_a, grad_w)
    t = float(case["temperature"])
    n, classes = case["n"], case["classes"]
    loss = torch.zeros(n, device=DEV, dtype=torch.float64)
    grad = None if case["grad"] == "none" else torch.zeros(n, classes, device=DEV, dtype=torch.float64)
    step = max(1, (1 << 27) // classes)
    for r in range(0, n, step):
        z = s["logits"][r:r + step].double() / t
        ids, w = s["ids"][r:r + step].long(), s["weight"][r:r + step].double()
        teacher = (s["top"][r:r + step].double() / t).masked_fill(ids < 0, -math.inf)
        log_p = teacher - torch.logsumexp(teacher, 1, keepdim=True)
        log_q = z - torch.logsumexp(z, 1, keepdim=True)
        empty = (ids < 0).all(1)
        w = w.masked_fill(empty, 0.0)
        terms = log_p.exp() * (log_p - log_q.gather(1, ids.clamp_min(0)))
        loss[r:r + step] = w * t * t * terms.masked_fill((ids < 0) | empty[:, None], 0.0).sum(1)
        if grad is not None:
            d = log_q.exp()
            d.scatter_add_(1, ids.clamp_min(0), -log_p.exp().masked_fill((ids < 0) | empty[:, None], 0.0))
            grad[r:r + step] = d * (w * t)[:, None]
    return loss if grad is None else (loss, grad)


# ---- what a pass cannot do without ---------------------------------------------------------------------------
def _distinct(n, rows):
    """Expected number of distinct rows among n ids of the power law above."""
    edges = np.unique(np.round(np.logspace(0, math.log10(rows + 1), 400)))
    width = edges[1:] - edges[:-1]
    mass = np.log(edges[1:] / edges[:-1]) / math.log(rows + 1.0)
    return float(np.sum(width * -np.expm1(-n * mass / width)))


def work(case):
    kind, n = case["kind"], case["n"]
    if kind in ("embed", "embed_grad"):
        dim, id_bytes = case["dim"], 8 if case["ids"] == "i64" else 4
        found = n * (15 / 16 if n >= 16 else 1.0)
        distinct = _distinct(found, case["rows"])
        if kind == "embed":
            return {"bytes": distinct * dim * SIZE[case["table"]] + n * (dim * SIZE[case["out"]] + id_bytes), "flops": n * dim}
        written = case["rows"] * dim * SIZE[case["out"]] * (2 if case["accumulate"] else 1)
        return {"bytes": found * dim * SIZE[case["grad"]] + n * id_bytes + written, "flops": found * dim}
    if kind in ("grouped", "grouped_grad"):
        k, m, size = case["d_in"], case["d_out"], SIZE[case["dtype"]]
        weights = min(case["groups"], n) * k * m
        if kind == "grouped":
            return {"bytes": n * k * size + weights * size + n * m * SIZE[case["out"]], "flops": 2.0 * n * k * m}
        seen = 2 if case["act"] == "relu" else 1
        grad_w = case["groups"] * k * m * SIZE[case["dw"]] * (2 if case["accumulate"] else 1)
        return {"bytes": n * (2 * k + seen * m) * size + weights * size + grad_w, "flops": 4.0 * n * k * m}
    kept = n * (1.0 - case["masked"])
    teacher = kept * case["k"] * (SIZE[case["top"]] + (8 if case["ids"] == "i64" else 4))
    logits = kept * case["classes"] * SIZE[case["logits"]]
    written = n * case["classes"] * SIZE[case["grad"]] if case["grad"] != "none" else 0
    return {"bytes": logits + teacher + written + n * 8, "flops": kept * case["classes"] * (6 if written else 4)}
