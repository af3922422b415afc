"""The work of asking how sure labels are, and of learning from a teacher's best classes, whose time is measured.

Propagated labels, or the logits of any model, are rows of one value per class.  ``rows`` says of each row what the log probabilities
of given classes are, how unsure the row is (its entropy) and which classes come first (``row_scores``); ``ask`` says the same of the
student's head, whose logits are not kept (``head_scores``).  A teacher's first classes with their logits are enough to learn from:
``learn`` is the divergence of the student from them, with its gradients (``head_distill``).  Heads have from two to 131,072 classes
(several sets of labels may share one head).  The plain forms are elementary torch operations in 32 bits.

Whole numbers come back from ``rows`` and ``ask`` (the first classes, of equal ones the lowest).  So that they do not hang on the order of a
sum, the inputs of ``ask`` lie on a grid on which every sum is exact in 32 bits; the other inputs are what random numbers give.
"""
import math

import torch

own = False

_TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}


def listed():
    return [
        # one row of logits that a service looks at: latency of one call
        dict(name="rows_one", op="rows", items=1, classes=1000, top=5, given=1, dtype="float32", probabilities=False),
        # propagated labels of a million vertices: which to ask about next, and what else they might be
        dict(name="rows_1m", op="rows", items=1000000, classes=50, top=4, given=0, dtype="float32", probabilities=True),
        # logits of a teacher with 100,003 classes, of which the first 32 are kept
        dict(name="rows_teacher", op="rows", items=4099, classes=100003, top=32, given=1, dtype="bfloat16", probabilities=False),
        # the student's answer for one item: latency
        dict(name="ask_one", op="ask", items=1, dim=256, classes=10007, top=5, given=1, dtype="bfloat16"),
        # 64 items and 131,072 classes: the head is read once
        dict(name="ask_64", op="ask", items=64, dim=1024, classes=131072, top=8, given=1, dtype="bfloat16"),
        # a batch of a tagging service: odd sizes, 29 classes
        dict(name="ask_20k", op="ask", items=20011, dim=200, classes=29, top=3, given=1, dtype="float16"),
        # a head in 32 bits, some candidates per item
        dict(name="ask_2k_32bit", op="ask", items=2003, dim=512, classes=10007, top=10, given=7, dtype="float32"),
        # a teacher's first classes for 8,192 items, made with its head
        dict(name="ask_8k", op="ask", items=8192, dim=1024, classes=32768, top=16, given=1, dtype="bfloat16"),
        # an update after one batch of vertices: few rows, a thousand classes
        dict(name="learn_128", op="learn", items=128, dim=128, classes=1000, kept=8, temperature=2.0, dtype="float16", grad="same"),
        # the labels of the 100,000-vertex graph: 64 dimensions, 10 classes, the first four of each row
        dict(name="learn_100k", op="learn", items=100000, dim=64, classes=10, kept=4, temperature=1.0, dtype="float32", grad="float32"),
        # a million rows of 50 classes, the first eight of each
        dict(name="learn_1m", op="learn", items=1000000, dim=256, classes=50, kept=8, temperature=1.0, dtype="bfloat16", grad="float32"),
        # a large step of training: 8,192 rows, 50,021 classes
        dict(name="learn_8k", op="learn", items=8192, dim=1024, classes=50021, kept=32, temperature=2.0, dtype="bfloat16", grad="same"),
    ]


def _log_uniform(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["rows", "rows", "ask", "ask", "ask", "learn", "learn", "learn"])
    dtype = rng.choice(["float32", "bfloat16", "float16"])
    classes = _log_uniform(rng, 2, 131072)
    if op == "rows":
        probabilities = rng.random() < 0.3
        items = min(_log_uniform(rng, 1, 1000003), 400000000 // classes)
        return dict(op=op, items=items, classes=classes, top=rng.randint(1, min(classes, 64)), given=rng.choice([0, 1, 1, 5]),
                    dtype="float32" if probabilities else dtype, probabilities=probabilities)
    dim = rng.choice([16, 50, 64, 128, 200, 256, 301, 512, 1000, 1024])
    if op == "ask":
        items = max(1, min(_log_uniform(rng, 1, 300007), 100000000 // dim, 270000000 // classes, 270000000000 // (classes * dim)))
        return dict(op=op, items=items, dim=dim, classes=classes, top=rng.randint(1, min(classes, 32)), given=rng.choice([0, 1, 1, 5]), dtype=dtype)
    kept = min(rng.choice([1, 2, 5, 8, 16, 32, 64]), classes)
    items = max(1, min(_log_uniform(rng, 1, 1000003), 256000000 // dim, 400000000 // classes, 400000000000 // (classes * dim)))
    return dict(op=op, items=items, dim=dim, classes=classes, kept=kept, temperature=rng.choice([1.0, 2.0, 3.0]), dtype=dtype,
                grad=rng.choice(["same", "float32"]))


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _given(n, c, count, g):
    """Classes that are asked about; some are padding."""
    if not count:
        return None
    ids = torch.randint(0, c, (n, count), generator=g, device="cuda", dtype=torch.int32)
    ids[torch.rand(n, count, generator=g, device="cuda") < 0.05] = -1
    return ids


def _grid(x, step):
    return torch.round(x / step) * step


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    op, dtype, n, c = case["op"], _TYPES[case["dtype"]], case["items"], case["classes"]
    state = dict(case)
    if op == "rows":
        x = torch.randn(n, c, generator=g, device="cuda")
        if case["probabilities"]:
            # propagated labels: unsure rows, and one-hot ones of labelled vertices
            x = torch.softmax(x.mul_(2.5), 1)
            seeds = torch.rand(n, generator=g, device="cuda") < 0.01
            x[seeds] = torch.nn.functional.one_hot(x[seeds].argmax(1), c).float()
        else:
            x.mul_(3.0)
            shut = torch.rand(c, generator=g, device="cuda") < 0.01  # classes that are not allowed
            shut[0] = False
            x[:, shut] = -math.inf
        state["x"] = x.to(dtype)
        state["ids"] = _given(n, c, case["given"], g)
        return state
    d = case["dim"]
    h = torch.randn(n, d, generator=g, device="cuda")
    weight = 2.0 / math.sqrt(d) * torch.randn(c, d, generator=g, device="cuda")
    bias = 0.1 * torch.randn(c, generator=g, device="cuda")
    if op == "ask":
        # 1/8 times 1/256: sums below 8,192 are exact
        state["h"], state["weight"], state["bias"] = _grid(h, 1 / 8).to(dtype), _grid(weight, 1 / 256).to(dtype), _grid(bias, 1 / 256)
        state["ids"] = _given(n, c, case["given"], g)
        return state
    state["h"], state["weight"], state["bias"] = h.to(dtype), weight.to(dtype), bias
    # a teacher's first classes: distinct, from the likeliest on, not as many for some rows
    k = case["kept"]
    at = torch.arange(k, device="cuda")
    first = torch.randint(0, c, (n, 1), generator=g, device="cuda")
    classes = ((first + at * max(1, c // k)) % c).to(torch.int32)
    length = 1 + torch.floor(k * torch.rand(n, 1, generator=g, device="cuda") * 1.5)
    state["kept_classes"] = torch.where(at < length, classes, torch.full_like(classes, -1))
    gaps = 0.6 * torch.rand(n, k, generator=g, device="cuda")
    state["kept_logits"] = (8.0 + torch.randn(n, 1, generator=g, device="cuda") - torch.cumsum(gaps, 1)).contiguous()
    r = torch.rand(n, generator=g, device="cuda")
    state["row_weight"] = torch.where(r < 0.05, torch.zeros_like(r), r)
    state["grad_scale"] = 1.0 / n
    return state


# ---- one pass --------------------------------------------------------------------------------------------------------

def run(state):
    return _own(state) if own else _PLAIN[state["op"]](state)


def _own(s):
    import paper_2604_06596_amd as P

    if s["op"] == "learn":
        loss, dh, dweight, dbias = P.head_distill(s["h"], s["weight"], s["bias"], s["kept_classes"], s["kept_logits"], temperature=s["temperature"],
                                                  row_weight=s["row_weight"], grad_scale=s["grad_scale"], dtype=_grad_type(s))
        return {"loss": loss, "dh": dh, "dweight": dweight, "dbias": dbias}
    if s["op"] == "rows":
        r = P.row_scores(s["x"], given=s["ids"], top=s["top"], probabilities=s["probabilities"])
    else:
        r = P.head_scores(s["h"], s["weight"], s["bias"], given=s["ids"], top=s["top"])
    return {"log_given": r.log_given, "entropy": r.entropy, "top": r.top, "log_top": r.log_top}


def _grad_type(s):
    return torch.float32 if s["grad"] == "float32" else _TYPES[s["dtype"]]


def _first(x, k):
    """The k largest of each row, of equal ones those of the lowest columns: keys of 64 bits, the value's order above the column's."""
    bits = (x + 0.0).view(torch.int32).long()
    key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits)
    key = (key << 32) + (x.shape[1] - 1 - torch.arange(x.shape[1], device="cuda"))
    return (x.shape[1] - 1 - (torch.topk(key, k, dim=1).values & 0xFFFFFFFF)).to(torch.int32)


def _plain_scores(s, order, log_p):
    p = torch.exp(log_p)
    entropy = -torch.where(p > 0, p * log_p, torch.zeros_like(p)).sum(1)
    top = _first(order, s["top"])
    out = {"log_given": None, "entropy": entropy, "top": top, "log_top": log_p.gather(1, top.long())}
    if s["ids"] is not None:
        out["log_given"] = torch.where(s["ids"] >= 0, log_p.gather(1, s["ids"].clamp(min=0).long()), torch.zeros((), device="cuda"))
    return out


def _plain_rows(s):
    x = s["x"].float()
    if s["probabilities"]:
        return _plain_scores(s, x, torch.log(x) - torch.log(x.sum(1, keepdim=True)))
    return _plain_scores(s, x, _log_softmax(x))


def _log_softmax(z):
    z = z - z.amax(1, keepdim=True)
    return z - torch.log(torch.exp(z).sum(1, keepdim=True))


def _plain_ask(s):
    z = s["h"].float() @ s["weight"].float().t().contiguous() + s["bias"]
    return _plain_scores(s, z, _log_softmax(z))


def _plain_learn(s):
    t = s["temperature"]
    z = s["h"].float() @ s["weight"].float().t().contiguous() + s["bias"]
    log_p = _log_softmax(z / t)
    kept = s["kept_classes"] >= 0
    at = s["kept_classes"].clamp(min=0).long()
    log_q = _log_softmax(torch.where(kept, s["kept_logits"] / t, torch.full_like(s["kept_logits"], -math.inf)))
    q = torch.exp(log_q)
    terms = torch.where(kept, q * (log_q - log_p.gather(1, at)), torch.zeros_like(q))
    loss = s["row_weight"] * (t * t) * terms.sum(1)
    dz = torch.exp(log_p).scatter_add_(1, at, -q) * (s["grad_scale"] * t * s["row_weight"])[:, None]
    dh = dz @ s["weight"].float()
    dweight = dz.t().contiguous() @ s["h"].float()
    return {"loss": loss, "dh": dh.to(s["h"].dtype), "dweight": dweight.to(_grad_type(s)), "dbias": dz.sum(0)}


_PLAIN = {"rows": _plain_rows, "ask": _plain_ask, "learn": _plain_learn}


# ---- what a pass cannot do without -----------------------------------------------------------------------------------

def work(case):
    n, c, size = case["items"], case["classes"], 4.0 if case["dtype"] == "float32" else 2.0
    if case["op"] == "learn":
        d, k = case["dim"], case["kept"]
        out = size * n * d + (4.0 if case["grad"] == "float32" else size) * c * d + 4.0 * (n + c)
        return {"bytes": size * (n + c) * d + 4.0 * c + n * (8.0 * k + 4.0) + out, "flops": 6.0 * n * c * d}
    out = n * (8.0 * case["top"] + 4.0 + 8.0 * case["given"])
    if case["op"] == "rows":
        return {"bytes": size * n * c + out, "flops": 8.0 * n * c}
    return {"bytes": size * (n + c) * case["dim"] + 4.0 * c + out, "flops": 2.0 * n * c * case["dim"]}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] != "learn":
        if case["op"] == "ask":
            z = torch.addmm(s["bias"].double(), s["h"].double(), s["weight"].double().t())
        else:
            z = s["x"].double()
            if case["probabilities"]:
                z = z.log_()
        z -= torch.logsumexp(z, 1, keepdim=True)
        order, column = torch.sort(z, dim=1, descending=True, stable=True)
        log_top, top = order[:, :case["top"]].contiguous(), column[:, :case["top"]].to(torch.int32)
        del column
        entropy = -torch.xlogy(order.exp(), order.exp()).sum(1)
        del order
        out = {"log_given": None, "entropy": entropy, "top": top, "log_top": log_top}
        if s["ids"] is not None:
            picked = torch.take_along_dim(z, s["ids"].long().remainder(case["classes"]), 1)
            picked[s["ids"] < 0] = 0.0
            out["log_given"] = picked
        return out
    t, h, W = case["temperature"], s["h"].double(), s["weight"].double()
    z = torch.addmm(s["bias"].double(), h, W.t()) / t
    lse = torch.logsumexp(z, 1, keepdim=True)
    row, column = torch.nonzero(s["kept_classes"] >= 0, as_tuple=True)
    u = torch.full(s["kept_logits"].shape, -math.inf, dtype=torch.float64, device="cuda")
    u[row, column] = s["kept_logits"].double()[row, column] / t
    log_q = (u - torch.logsumexp(u, 1, keepdim=True))[row, column]
    classes = s["kept_classes"][row, column].long()
    gap = log_q.exp() * (log_q - z[row, classes] + lse[row, 0])
    loss = torch.zeros(case["items"], dtype=torch.float64, device="cuda").index_add_(0, row, gap)
    z = z.sub_(lse).exp_()
    z.index_put_((row, classes), -log_q.exp(), accumulate=True)
    r = s["row_weight"].double()
    z *= (s["grad_scale"] * t * r)[:, None]
    return {"loss": t * t * r * loss, "dh": z @ W, "dweight": (h.t() @ z).t().contiguous(), "dbias": z.sum(0)}
