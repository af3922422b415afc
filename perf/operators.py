"""The work of training and asking a student of propagated labels, whose time is measured.

Label propagation gives the vertices of a graph their class distributions.  A student learns them, so that items outside
the graph have labels too: the rows of an item's tokens in a table are added up with the tokens' weights (``embed``), a head
with one row per class turns the sum into a distribution (``answer``, ``loss``), and the gradients (``loss``, ``embed_grad``)
move table and head by AdamW (``adamw``).  The plain forms are elementary torch operations in 32 bits.

Token ids follow a law of 1 / (id + 10), as words do once the most frequent are left out; items have lengths around a mean,
none at all now and then; some tokens are padding (negative ids).
"""
import math
import random as _random

import numpy as np
import torch

own = False

_TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
_HEAD = 10.0  # ids i are drawn with a probability that falls as 1 / (i + _HEAD)
_BLOCK = 256  # elements of an 8-bit state that share a scale


def listed():
    return [
        # a service embeds the tokens of one item that has just arrived: latency of one call
        dict(name="embed_item", op="embed", rows=30011, dim=64, items=1, mean_len=37.0, dtype="float32"),
        # a batch of a tagging service: 20,011 short texts
        dict(name="embed_20k", op="embed", rows=100003, dim=128, items=20011, mean_len=60.0, dtype="bfloat16"),
        # one row per token, scaled, a tenth of them padding (items as sequences of tokens, not as sums)
        dict(name="embed_rows", op="embed", rows=250007, dim=1000, items=65536, mean_len=0.0, dtype="float16"),
        # a large step of training: 131,072 texts of 64 tokens, a table of a million rows
        dict(name="embed_131k", op="embed", rows=1000000, dim=256, items=131072, mean_len=64.0, dtype="bfloat16"),
        # the table's gradient for some thousand single tokens (an update after one batch of vertices)
        dict(name="grad_rows_4k", op="embed_grad", rows=30011, dim=128, items=4099, mean_len=0.0, dtype="float32"),
        # the table's gradient in the large step of training
        dict(name="grad_131k", op="embed_grad", rows=1000000, dim=256, items=131072, mean_len=64.0, dtype="bfloat16"),
        # the answer for one item: latency
        dict(name="answer_one", op="answer", items=1, dim=64, classes=10, dtype="float32"),
        # answers for the items of a graph that are no longer kept in it: odd sizes, 29 classes
        dict(name="answer_300k", op="answer", items=300007, dim=200, classes=29, dtype="float16"),
        # loss and gradients on the labels of the 100,000-vertex graph: 64 dimensions, 10 classes
        dict(name="loss_100k", op="loss", items=100000, dim=64, classes=10, dtype="float32", hard=False),
        # loss and gradients on a million rows of 50 classes
        dict(name="loss_1m", op="loss", items=1000000, dim=256, classes=50, dtype="bfloat16", hard=False),
        # one optimizer step over sixty tensors of all sizes, 24M elements, 32-bit states
        dict(name="adamw_60", op="adamw", tensors=60, total=24000000, bits=32, dtype="float32", copy=False),
        # one optimizer step over a table of a million rows of 256 and its head, 8-bit states, gradients and copy in bfloat16
        dict(name="adamw_table_8bit", op="adamw", tensors=3, total=256012850, bits=8, dtype="bfloat16", copy=True),
    ]


def _log_uniform(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["embed", "embed", "embed_grad", "embed_grad", "answer", "loss", "loss", "adamw", "adamw"])
    dtype = rng.choice(["float32", "bfloat16", "float16"])
    if op in ("embed", "embed_grad"):
        dim = rng.choice([16, 64, 100, 128, 200, 256, 333, 512, 1000, 1024])
        rows = min(_log_uniform(rng, 1009, 1000003), 256000000 // dim)
        if rng.random() < 0.3:
            items, mean_len = min(_log_uniform(rng, 1, 131071), 64000000 // dim), 0.0
        else:
            mean_len = round(math.exp(rng.uniform(0.0, math.log(200.0))), 1)
            items = min(_log_uniform(rng, 1, 131071), max(1, int(1.0e9 / dim / mean_len)))
        return dict(op=op, rows=rows, dim=dim, items=items, mean_len=mean_len, dtype=dtype)
    if op in ("answer", "loss"):
        dim = rng.choice([16, 50, 64, 128, 200, 256, 301, 512])
        classes = rng.choice([2, 3, 4, 10, 17, 29, 50, 64])
        items = min(_log_uniform(rng, 1, 1000003), 100000000 // dim)
        case = dict(op=op, items=items, dim=dim, classes=classes, dtype=dtype)
        return dict(case, hard=rng.random() < 0.4) if op == "loss" else case
    return dict(op=op, tensors=rng.randint(1, 60), total=_log_uniform(rng, 1009, 128000000), bits=rng.choice([8, 32]),
                dtype=rng.choice(["float32", "bfloat16"]), copy=rng.random() < 0.5)


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _tokens(case, g):
    """ids, offsets (None: one row per token) and weights of the case's items."""
    items, mean = case["items"], case["mean_len"]
    if mean:
        u = torch.rand(items, generator=g, device="cuda")
        lengths = torch.floor(2.0 * mean * u + 0.5).to(torch.int64)  # 0 .. 2 * mean
        offsets = torch.zeros(items + 1, dtype=torch.int64, device="cuda")
        torch.cumsum(lengths, 0, out=offsets[1:])
        count = int(offsets[-1])
    else:
        offsets, count = None, items
    u = torch.rand(count, generator=g, device="cuda", dtype=torch.float64)
    ids = torch.floor(_HEAD * torch.exp(u * math.log((case["rows"] + _HEAD) / _HEAD)) - _HEAD)
    ids = ids.clamp(0, case["rows"] - 1).to(torch.int32)
    ids[torch.rand(count, generator=g, device="cuda") < (0.02 if mean else 0.1)] = -1
    weights = 0.1 + torch.rand(count, generator=g, device="cuda") if mean else None
    return ids, offsets, weights


def _sizes(case):
    """Elements of each tensor: the table first, then sizes spread over their logarithm."""
    if case["tensors"] == 3 and case["total"] > 50 * 257:
        return [case["total"] - 50 * 257, 50 * 256, 50]
    rng = _random.Random(case["total"] * 64 + case["tensors"])
    share = [math.exp(rng.uniform(0.0, 7.0)) for _ in range(case["tensors"])]
    return [max(1, int(case["total"] * s / sum(share))) for s in share]


def _flat(sizes, unit):
    """Offsets of tensors in one flat array, each on a multiple of `unit`."""
    at, total = [], 0
    for n in sizes:
        at.append(total)
        total += -(-n // unit) * unit
    return at, total


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    op, dtype = case["op"], _TYPES[case["dtype"]]
    state = dict(case)
    if op in ("embed", "embed_grad"):
        state["ids"], state["offsets"], state["weights"] = _tokens(case, g)
        state["scale"] = math.sqrt(case["dim"]) if state["offsets"] is None else 0.125
        if op == "embed":
            state["table"] = (0.05 * torch.randn(case["rows"], case["dim"], generator=g, device="cuda")).to(dtype)
        else:
            state["grad"] = torch.randn(case["items"], case["dim"], generator=g, device="cuda").to(dtype)
    elif op in ("answer", "loss"):
        n, d, c = case["items"], case["dim"], case["classes"]
        state["h"] = torch.randn(n, d, generator=g, device="cuda").to(dtype)
        state["weight"] = (2.0 / math.sqrt(d) * torch.randn(c, d, generator=g, device="cuda")).to(dtype)
        state["bias"] = 0.1 * torch.randn(c, generator=g, device="cuda")
        if op == "loss":
            q = torch.softmax(2.5 * torch.randn(n, c, generator=g, device="cuda"), 1)
            hard = q.argmax(1).to(torch.int32)
            if case["hard"]:
                hard[torch.rand(n, generator=g, device="cuda") < 0.05] = -1
                state["target"], state["row_weight"] = hard, None
            else:
                seeds = torch.rand(n, generator=g, device="cuda") < 0.01  # labelled vertices: one-hot rows
                state["target"] = torch.where(seeds[:, None], torch.nn.functional.one_hot(hard.long(), c).float(), q).contiguous()
                r = torch.rand(n, generator=g, device="cuda")
                state["row_weight"] = torch.where(r < 0.05, torch.zeros_like(r), r)
            state["grad_scale"] = 1.0 / n
    else:
        sizes = _sizes(case)
        at, total = _flat(sizes, _BLOCK)
        cut = lambda flat: [flat[a:a + n] for a, n in zip(at, sizes)]  # noqa: E731
        flat = {"param": 0.05 * torch.randn(total, generator=g, device="cuda"),
                "grad": (0.01 * torch.randn(total, generator=g, device="cuda")).to(dtype)}
        flat["copy"] = flat["param"].to(torch.bfloat16) if case["copy"] else None
        m = 0.003 * torch.randn(total, generator=g, device="cuda")
        r = 0.01 * torch.exp(0.5 * torch.randn(total, generator=g, device="cuda"))
        if case["bits"] == 8:
            scales = lambda x: torch.exp2(torch.floor(torch.log2(x.abs().view(-1, _BLOCK).amax(1))) - 7.0)  # noqa: E731
            flat["m_scale"], flat["r_scale"] = scales(m), scales(r)
            flat["m"] = (m.view(-1, _BLOCK) / flat["m_scale"][:, None]).view(-1).to(torch.float8_e4m3fn)
            flat["r"] = (r.view(-1, _BLOCK) / flat["r_scale"][:, None]).view(-1).to(torch.float8_e4m3fn)
            blocks = lambda s: [s[a // _BLOCK:a // _BLOCK + -(-n // _BLOCK)] for a, n in zip(at, sizes)]  # noqa: E731
            state["states"] = list(zip(cut(flat["m"]), cut(flat["r"]), blocks(flat["m_scale"]), blocks(flat["r_scale"])))
        else:
            flat["m"], flat["v"] = m, r * r
            state["states"] = list(zip(cut(flat["m"]), cut(flat["v"])))
        state["flat"] = flat
        state["params"], state["grads"] = cut(flat["param"]), cut(flat["grad"])
        state["copies"] = cut(flat["copy"]) if case["copy"] else None
        state["decay"] = [0.01 if k % 2 == 0 else 0.0 for k in range(len(sizes))]
        state["step"], state["seed"] = 10, int(seed) % 65521
    return state


# ---- one pass --------------------------------------------------------------------------------------------------------

def run(state):
    return _own(state) if own else _PLAIN[state["op"]](state)


def _own(s):
    import paper_2604_06596_amd as P

    op = s["op"]
    if op == "embed":
        return P.embed(s["table"], s["ids"], s["offsets"], s["weights"], s["scale"])
    if op == "embed_grad":
        return P.embed_grad(s["grad"], s["ids"], s["rows"], s["offsets"], s["weights"], s["scale"])
    if op == "answer":
        return P.head_labels(s["h"], s["weight"], s["bias"], hard=False)[0]
    if op == "loss":
        loss, dh, dweight, dbias = P.head_loss(s["h"], s["weight"], s["bias"], s["target"], row_weight=s["row_weight"],
                                               grad_scale=s["grad_scale"])
        return {"loss": loss, "dh": dh, "dweight": dweight, "dbias": dbias}
    s["step"] += 1
    P.adamw_step(s["params"], s["grads"], s["states"], step=s["step"], lr=1e-3, betas=(0.9, 0.999), eps=1e-8,
                 weight_decay=s["decay"], copies=s["copies"], seed=s["seed"])
    return {k: v for k, v in s["flat"].items() if k != "grad"}


def _bags(ids, offsets):
    """The item of each token."""
    at = torch.arange(len(ids), device="cuda")
    return at if offsets is None else torch.searchsorted(offsets, at, right=True) - 1


def _factors(s):
    """scale * weight of each token, nothing for padding."""
    w = torch.full((len(s["ids"]),), s["scale"], device="cuda") if s["weights"] is None else s["scale"] * s["weights"]
    return torch.where(s["ids"] >= 0, w, torch.zeros_like(w))


def _plain_embed(s):
    rows = s["table"].index_select(0, s["ids"].clamp(min=0).long()).float() * _factors(s)[:, None]
    if s["offsets"] is not None:
        out = torch.zeros(s["items"], s["dim"], device="cuda")
        rows = out.index_add_(0, _bags(s["ids"], s["offsets"]), rows)
    return rows.to(s["table"].dtype)


def _plain_embed_grad(s):
    rows = s["grad"].index_select(0, _bags(s["ids"], s["offsets"])).float() * _factors(s)[:, None]
    out = torch.zeros(s["rows"], s["dim"], device="cuda")
    return out.index_add_(0, s["ids"].clamp(min=0).long(), rows)


def _plain_softmax(s):
    z = s["h"].float() @ s["weight"].float().t().contiguous() + s["bias"]
    z = z - z.amax(1, keepdim=True)
    e = torch.exp(z)
    total = e.sum(1, keepdim=True)
    return z, e / total, torch.log(total)


def _plain_answer(s):
    return _plain_softmax(s)[1]


def _plain_loss(s):
    z, p, lse = _plain_softmax(s)
    if s["target"].dtype == torch.int32:
        r = (s["target"] >= 0).float()
        q = (torch.arange(s["classes"], device="cuda")[None, :] == s["target"][:, None]).float()
    else:
        r, q = s["row_weight"], s["target"]
    loss = r * (q * (lse - z)).sum(1)
    dz = (s["grad_scale"] * r)[:, None] * (q.sum(1, keepdim=True) * p - q)
    dh = dz @ s["weight"].float()
    dweight = dz.t().contiguous() @ s["h"].float()
    return {"loss": loss, "dh": dh.to(s["h"].dtype), "dweight": dweight, "dbias": dz.sum(0)}


def _mix(x):
    """32 bits out of 32 bits, held in int64: shifts and odd factors (the fractions of the golden ratio and of the root of two)."""
    x = x ^ (x >> 16)
    x = (x * 0x9E3779B9) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0x6A09E667) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _to_8_bits(x, dither, keep):
    """Non-negative x as float8_e4m3fn codes with a power-of-two scale per block, rounded up where the 16-bit dither says so.
    keep: what is not zero stays so."""
    padded = torch.nn.functional.pad(x, (0, -len(x) % _BLOCK)).view(-1, _BLOCK)
    top = padded.amax(1).view(torch.int32) >> 23
    scale = torch.where(top >= 8, (top - 7) << 23, torch.zeros_like(top)).view(torch.float32)
    inverse = torch.where(top >= 8, (261 - top) << 23, torch.zeros_like(top)).view(torch.float32)
    y = (padded * inverse[:, None]).view(-1)[:len(x)]
    normal = ((y.view(torch.int32) + (dither.to(torch.int32) << 4)) >> 20) - (120 << 3)
    small = torch.floor(y * 512.0 + dither.float() * 2.0 ** -16).to(torch.int32)
    code = torch.where(y >= 2.0 ** -6, normal, small)
    if keep:
        code = torch.where((x > 0) & (inverse[:, None].expand(-1, _BLOCK).reshape(-1)[:len(x)] > 0), code.clamp(min=1), code)
    return code.to(torch.uint8), scale


def _plain_adamw(s):
    s["step"] += 1
    t, lr, b1, b2, eps = s["step"], 1e-3, 0.9, 0.999, 1e-8
    step_size, root = lr / (1.0 - b1 ** t), 1.0 / math.sqrt(1.0 - b2 ** t)
    for k, (p, g, st) in enumerate(zip(s["params"], s["grads"], s["states"])):
        g = g.float()
        if s["bits"] == 8:
            wide = lambda code, scale: code.float() * scale.repeat_interleave(_BLOCK)[:len(p)]  # noqa: E731
            m, r = wide(st[0], st[2]), wide(st[1], st[3])
            v = r * r
        else:
            m, v = st
        m = m * b1 + g * (1.0 - b1)
        v = v * b2 + (g * g) * (1.0 - b2)
        r = torch.sqrt(v)
        p.copy_(p * (1.0 - lr * s["decay"][k]) - step_size * (m / (r * root + eps)))
        if s["bits"] == 8:
            key = _mix(_mix(_mix(s["seed"]) ^ t) ^ k)
            h = _mix(torch.arange(len(p), device="cuda") ^ key)
            code, scale = _to_8_bits(m.abs(), h & 0xFFFF, False)
            st[0].view(torch.uint8).copy_(code | (m.view(torch.int32) < 0).to(torch.uint8) << 7)
            st[2].copy_(scale)
            code, scale = _to_8_bits(r, h >> 16, True)
            st[1].view(torch.uint8).copy_(code)
            st[3].copy_(scale)
        else:
            st[0].copy_(m)
            st[1].copy_(v)
        if s["copies"] is not None:
            s["copies"][k].copy_(p)
    return {k: v for k, v in s["flat"].items() if k != "grad"}


_PLAIN = {"embed": _plain_embed, "embed_grad": _plain_embed_grad, "answer": _plain_answer, "loss": _plain_loss, "adamw": _plain_adamw}


# ---- what a pass cannot do without -----------------------------------------------------------------------------------

def _distinct(case, count):
    """How many rows of the table `count` tokens of the law above name, on average."""
    i = np.arange(case["rows"], dtype=np.float64) + _HEAD
    chance = np.log1p(1.0 / i) / math.log((case["rows"] + _HEAD) / _HEAD)
    return float(np.sum(-np.expm1(-count * chance)))


def work(case):
    op, size = case["op"], 4 if case["dtype"] == "float32" else 2
    if op in ("embed", "embed_grad"):
        count = case["items"] * (case["mean_len"] or 1.0)
        lists = 4.0 * count + (8.0 * case["items"] + 4.0 * count if case["mean_len"] else 0.0)
        flops = 2.0 * count * case["dim"]
        if op == "embed":
            return {"bytes": lists + size * case["dim"] * (_distinct(case, count) + case["items"]), "flops": flops}
        return {"bytes": lists + case["dim"] * (size * case["items"] + 4.0 * case["rows"]), "flops": flops}
    if op in ("answer", "loss"):
        n, d, c = case["items"], case["dim"], case["classes"]
        data = float(size) * (n * d + c * d) + 4.0 * c
        if op == "answer":
            return {"bytes": data + 4.0 * n * c, "flops": 2.0 * n * d * c}
        target = 4.0 * n if case["hard"] else 4.0 * n * c + 4.0 * n
        return {"bytes": data + target + float(size) * n * d + 4.0 * (c * d + c + n), "flops": 6.0 * n * d * c}
    total = float(sum(_sizes(case)))
    states = 4.0 + 16.0 / _BLOCK if case["bits"] == 8 else 16.0
    return {"bytes": total * (8.0 + size + states + (2.0 if case["copy"] else 0.0)), "flops": 15.0 * total}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("embed", "embed_grad"):
        ids = s["ids"].long()
        real = ids >= 0
        if s["offsets"] is None:
            item = torch.arange(len(ids), device="cuda")
        else:
            item = torch.repeat_interleave(torch.arange(case["items"], device="cuda"), s["offsets"].diff())
        w = torch.full_like(ids, s["scale"], dtype=torch.float64) if s["weights"] is None else s["scale"] * s["weights"].double()
        ids, item, w = ids[real], item[real], w[real]
        source, to, frm, out_rows = (s["table"], item, ids, case["items"]) if op == "embed" else (s["grad"], ids, item, case["rows"])
        order = torch.argsort(to, stable=True)
        crow = torch.searchsorted(to[order], torch.arange(out_rows + 1, device="cuda"))
        A = torch.sparse_csr_tensor(crow, frm[order], w[order], (out_rows, source.shape[0]))
        return A @ source.double()
    if op in ("answer", "loss"):
        h, W = s["h"].double(), s["weight"].double()
        z = torch.addmm(s["bias"].double(), h, W.t())
        log_p = z - torch.logsumexp(z, 1, keepdim=True)
        if op == "answer":
            return log_p.exp()
        if case["hard"]:
            r = torch.where(s["target"] >= 0, 1.0, 0.0).double()
            q = torch.zeros_like(z).scatter_(1, s["target"].long().clamp(min=0)[:, None], 1.0)
        else:
            r, q = s["row_weight"].double(), s["target"].double()
        dz = s["grad_scale"] * r[:, None] * (q.sum(1, keepdim=True) * log_p.exp() - q)
        return {"loss": -r * (q * log_p).sum(1), "dh": dz @ W, "dweight": (h.t() @ dz).t().contiguous(), "dbias": dz.sum(0)}
    t = s["step"] + 1
    out = {k: None for k in s["flat"] if k != "grad"}
    flat = {k: None if v is None else v.double() if v.dtype != torch.float8_e4m3fn else v.float().double() for k, v in s["flat"].items()}
    m, v = flat["m"], flat["v"] if case["bits"] == 32 else (flat["r"].view(-1, _BLOCK) * flat["r_scale"][:, None]).view(-1) ** 2
    if case["bits"] == 8:
        m = (m.view(-1, _BLOCK) * flat["m_scale"][:, None]).view(-1)
    inside = torch.zeros(len(m), dtype=torch.bool, device="cuda")
    decay = torch.zeros(len(m), dtype=torch.float64, device="cuda")
    for p, d in zip(s["params"], s["decay"]):
        at = p.storage_offset()
        inside[at:at + len(p)] = True
        decay[at:at + len(p)] = d
    g = flat["grad"]
    m1 = 0.9 * m + 0.1 * g
    v1 = 0.999 * v + 0.001 * g * g
    moved = flat["param"] - 1e-3 * (decay * flat["param"] + (m1 / (1 - 0.9 ** t)) / ((v1 / (1 - 0.999 ** t)).sqrt() + 1e-8))
    out["param"] = torch.where(inside, moved, flat["param"])
    if case["copy"]:
        out["copy"] = out["param"]
    if case["bits"] == 32:
        out["m"], out["v"] = torch.where(inside, m1, m), torch.where(inside, v1, v)
    return out
