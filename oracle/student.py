"""Plain definitions, in 64 bits, of what a student of propagated labels computes (numpy, loops over items and tensors).

``embed`` / ``embed_grad``: weighted sums of token rows and the table's gradient.  ``head`` / ``head_loss``: class
distributions, cross entropy and its gradients.  ``adamw``: one step, and the 8-bit format of its states.
Next to each result stands the sum of the magnitudes that went into it, which error bounds are made of.
"""
import numpy as np


def items_of(count, items, offsets):
    """The item of each token, -1 for a token that is in none."""
    if offsets is None:
        return np.arange(count)
    item = np.full(count, -1, dtype=np.int64)
    for b in range(items):
        item[max(int(offsets[b]), 0):max(int(offsets[b + 1]), 0)] = b
    return item


def _sum_rows(rows, key, source, factor, out_rows):
    out = np.zeros((out_rows, rows.shape[1]))
    magnitude = np.zeros_like(out)
    terms = np.zeros(out_rows, dtype=np.int64)
    for k, s, f in zip(key, source, factor):
        if 0 <= k < out_rows and 0 <= s < len(rows):
            out[k] += f * rows[s]
            magnitude[k] += np.abs(f * rows[s])
            terms[k] += 1
    return out, magnitude, terms


def embed(table, ids, offsets=None, weights=None, scale=1.0):
    """(out, sums of magnitudes, numbers of terms)."""
    items = len(ids) if offsets is None else len(offsets) - 1
    f = scale * (np.ones(len(ids)) if weights is None else np.asarray(weights, dtype=np.float64))
    return _sum_rows(np.asarray(table, dtype=np.float64), items_of(len(ids), items, offsets), ids, f, items)


def embed_grad(grad, ids, num_rows, offsets=None, weights=None, scale=1.0):
    """(gradient of the table, sums of magnitudes, numbers of terms)."""
    f = scale * (np.ones(len(ids)) if weights is None else np.asarray(weights, dtype=np.float64))
    return _sum_rows(np.asarray(grad, dtype=np.float64), ids, items_of(len(ids), len(grad), offsets), f, num_rows)


def head(h, weight, bias=None):
    """(logits, soft labels, hard labels).  A row whose logits are all -infinity is 1/C and class 0."""
    with np.errstate(invalid="ignore", over="ignore"):
        z = np.asarray(h, dtype=np.float64) @ np.asarray(weight, dtype=np.float64).T
        if bias is not None:
            z = z + np.asarray(bias, dtype=np.float64)
        top = z.max(axis=1, keepdims=True)
        e = np.where(np.isneginf(z), 0.0, np.exp(z - np.where(np.isneginf(top), 0.0, top)))
        total = e.sum(axis=1, keepdims=True)
        soft = np.where(total == 0.0, 1.0 / z.shape[1], e / total)
    return z, soft, np.argmax(np.where(np.isnan(z), -np.inf, z), axis=1)


def head_loss(h, weight, bias, soft=None, hard=None, row_weight=None, grad_scale=1.0):
    """dict of loss, dh, dweight, dbias, dz, and left_out (rows that take no part)."""
    h, weight = np.asarray(h, dtype=np.float64), np.asarray(weight, dtype=np.float64)
    n, classes = len(h), len(weight)
    r = np.ones(n) if row_weight is None else np.asarray(row_weight, dtype=np.float64)
    out = (r == 0.0)
    if hard is not None:
        out = out | (hard < 0) | (hard >= classes)
        soft = np.zeros((n, classes))
        soft[np.arange(n)[~out], np.asarray(hard)[~out]] = 1.0
    soft = np.where(out[:, None], 0.0, np.asarray(soft, dtype=np.float64))
    z, p, _ = head(np.where(out[:, None], 0.0, h), weight, bias)
    out = out | np.isneginf(z).all(axis=1)
    top = np.where(out, 0.0, z.max(axis=1, initial=-np.inf))
    with np.errstate(divide="ignore", invalid="ignore"):
        lse = np.log(np.exp(z - top[:, None]).sum(axis=1)) + top
        loss = np.where(soft != 0.0, soft * (lse[:, None] - z), 0.0).sum(axis=1)
    dz = grad_scale * r[:, None] * (soft.sum(axis=1, keepdims=True) * p - soft)
    dz[out] = 0.0
    return {"loss": np.where(out, 0.0, r * loss), "dh": dz @ weight, "dweight": dz.T @ np.where(out[:, None], 0.0, h), "dbias": dz.sum(axis=0),
            "dz": dz, "left_out": out, "soft": p, "logits": z, "target": soft}


# ---- AdamW --------------------------------------------------------------------------------------------------------------

STATE_BLOCK = 256
FORMAT = np.array([(m / 512.0 if e == 0 else (1 + m / 8.0) * 2.0 ** (e - 7)) for e in range(16) for m in range(8)])  # codes 0 .. 127


def adamw(param, grad, m, v, step, lr, beta1, beta2, eps, weight_decay, grad_scale=1.0):
    """(param, m, v) after one step."""
    g = grad_scale * np.asarray(grad, dtype=np.float64)
    m = beta1 * np.asarray(m, dtype=np.float64) + (1.0 - beta1) * g
    v = beta2 * np.asarray(v, dtype=np.float64) + (1.0 - beta2) * g * g
    update = (m / (1.0 - beta1 ** step)) / (np.sqrt(v) / np.sqrt(1.0 - beta2 ** step) + eps)
    return np.asarray(param, dtype=np.float64) * (1.0 - lr * weight_decay) - lr * update, m, v


def state_scales(x):
    """The power of two of each block, so that its largest magnitude lies in 128 .. 256 of the format (0: below 2^-119)."""
    scales = []
    for at in range(0, len(x), STATE_BLOCK):
        top = np.abs(x[at:at + STATE_BLOCK]).max()
        scales.append(0.0 if top < 2.0 ** -119 else 2.0 ** (np.floor(np.log2(top)) - 7))
    return np.array(scales)


def state_values(codes, scales):
    """What 8-bit codes stand for."""
    codes = np.asarray(codes).astype(np.int64)
    value = FORMAT[codes & 127] * np.where(codes & 128, -1.0, 1.0)
    return value * np.repeat(scales, STATE_BLOCK)[:len(codes)]


def state_neighbours(y):
    """The format's largest value not above y >= 0 and its smallest not below, in units of the scale."""
    at = np.searchsorted(FORMAT, y, side="right") - 1
    low = FORMAT[np.clip(at, 0, 126)]
    return low, np.where(low == y, y, FORMAT[np.clip(at + 1, 0, 126)])


# ---- scores and learning from a teacher's first classes ------------------------------------------------------------------

def scores(x, probabilities=False):
    """(log probabilities, entropy, order of the classes) of rows of logits, or of probabilities."""
    x = np.asarray(x, dtype=np.float64)
    with np.errstate(divide="ignore", invalid="ignore"):
        z = np.log(x) if probabilities else x
        top = z.max(axis=1, keepdims=True)  # not a number where one is
        finite = np.where(np.isneginf(top), 0.0, top)
        log_s = np.log(np.where(np.isneginf(z), 0.0, np.exp(z - finite)).sum(axis=1, keepdims=True))
        log_p = np.where(np.isneginf(top), -np.log(z.shape[1]), (z - finite) - log_s)
        p = np.exp(log_p)
        entropy = -np.where(p == 0.0, 0.0, p * np.where(p == 0.0, 0.0, log_p)).sum(axis=1)
    order = np.argsort(np.where(np.isnan(x), np.inf, -x), axis=1, kind="stable")
    return log_p, entropy, order


def distill(h, weight, bias, classes, logits, temperature=1.0, row_weight=None, grad_scale=1.0):
    """dict of loss, dh, dweight, dbias, dz, left_out, target (dense), soft (at the temperature), logits (divided by it)."""
    h, weight = np.asarray(h, dtype=np.float64), np.asarray(weight, dtype=np.float64)
    n, count = len(h), len(weight)
    r = np.ones(n) if row_weight is None else np.asarray(row_weight, dtype=np.float64)
    target, entropy = np.zeros((n, count)), np.zeros(n)
    out = r == 0.0
    for i in range(n):
        real = (classes[i] >= 0) & (classes[i] < count)
        u = np.asarray(logits[i], dtype=np.float64)[real] / temperature
        if out[i] or len(u) == 0 or np.isneginf(u).all():
            out[i] = True
            continue
        with np.errstate(invalid="ignore"):
            e = np.exp(u - u.max())
            q = e / e.sum()
            np.add.at(target[i], classes[i][real], q)
            q = target[i]  # of a class, however many entries name it
            entropy[i] = np.where(q == 0.0, 0.0, q * np.log(np.where(q == 0.0, 1.0, q))).sum()
    z, p, _ = head(np.where(out[:, None], 0.0, h), weight, bias)
    out = out | np.isneginf(z).all(axis=1)
    z = z / temperature
    top = np.where(out, 0.0, z.max(axis=1, initial=-np.inf))
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.exp(z - top[:, None])
        total = e.sum(axis=1)
        p = e / total[:, None]
        lse = np.log(total) + top
        loss = entropy + np.where(target != 0.0, target * (lse[:, None] - z), 0.0).sum(axis=1)
        dz = grad_scale * r[:, None] * temperature * (np.where(np.isnan(target).any(axis=1, keepdims=True), np.nan, p) - target)
    dz[out] = 0.0
    return {"loss": np.where(out, 0.0, r * temperature ** 2 * loss), "dh": np.where(out[:, None], 0.0, dz @ weight),
            "dweight": dz.T @ np.where(out[:, None], 0.0, h), "dbias": dz.sum(axis=0), "dz": dz, "left_out": out, "target": target, "soft": p,
            "logits": z, "lse": lse}
