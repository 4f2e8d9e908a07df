"""The operators of a serving step (tokens placed, looked up, adapted, drawn), plainly and in 64 bits on the CPU.  Shares no code with the library."""
import math

import numpy as np
import torch

from operators_plain import wide


def place(pages, page_size, lengths, new, free, n_free, n_tokens, ends=None):
    """(slots, starts, lengths, owners, n_free, pages, free, told) as lists, one sequence behind the other.  told: how many sequences got nothing though they asked for something
    they could not have."""
    table, free, lengths = [list(r) for r in pages], list(free), list(lengths)
    width = len(table[0]) if table else 0
    stack = free[:n_free]
    for s, e in enumerate(ends or []):
        if e:
            stack += table[s][:math.ceil(lengths[s] / page_size)]
            lengths[s] = 0
    free[:len(stack)] = stack
    top, upto, told, total = len(stack), 0, 0, 0
    slots, owners, starts = [-1] * n_tokens, [-1] * n_tokens, [0]
    for s, n in enumerate(new):
        more = max(n, 0)
        start, total = total, total + more
        starts.append(min(total, n_tokens))
        for t in range(start, min(total, n_tokens)):
            owners[t] = s
        if n < 0 or lengths[s] < 0 or lengths[s] + more > width * page_size or total > n_tokens:
            told += 1
            continue
        need = math.ceil((lengths[s] + more) / page_size) - math.ceil(lengths[s] / page_size)
        upto += need
        if need and upto > top:
            told += 1
            continue
        for j in range(more):
            at = lengths[s] + j
            if at % page_size == 0:
                table[s][at // page_size] = stack.pop()
            slots[start + j] = table[s][at // page_size] * page_size + at % page_size
        lengths[s] += more
    return slots, starts, lengths, owners, len(stack), table, free, told


def embed(tokens, weight, zero_point=0, row_scales=None, scale=1.0):
    """In 32 bits, operation by operation, which is what is asked for: one rounding of scale * row_scale, one of the product."""
    w = weight.cpu().float()
    by = torch.full((len(w),), scale, dtype=torch.float32)
    if row_scales is not None:
        by = row_scales.cpu() * by
    out = torch.zeros(len(tokens), w.shape[1])
    for i, t in enumerate(tokens.tolist()):
        if 0 <= t < len(w):
            out[i] = by[t] * (w[t] - zero_point)
    return out


def adapt(base, x, a, b, ids, x_scales=None, scales=None, activation="none", mul=None, residual=None, short=True):
    """(y, error): sums of 32 bits are off by 2^-24 of the sum of sizes for each addition; h by 2^-18 with `short`; scales and the epilogue round a few times, no
    activation is steeper than 1.13, and gelu's erf is good to 1.5e-7."""
    z = wide(base)
    error = z.abs() * 2.0 ** -23
    k, rank = x.shape[1], a.shape[1]
    for r, i in enumerate(ids.tolist()):
        if not 0 <= i < len(a):
            continue
        by = (float(scales[i]) if scales is not None else 1.0) * (float(x_scales[r]) if x_scales is not None else 1.0)
        wa, wb = wide(a[i]), wide(b[i])
        h = wa @ wide(x[r]) * by
        h_error = wa.abs() @ wide(x[r]).abs() * abs(by) * (k + 8) * 2.0 ** -24 + h.abs() * (2.0 ** -18 if short else 0.0)
        z[r] += wb @ h
        error[r] += wb.abs() @ h_error + wb.abs() @ h.abs() * (3 * rank + 8) * 2.0 ** -24 + z[r].abs() * 2.0 ** -23
    y = {"none": lambda t: t, "relu": torch.relu, "gelu": lambda t: 0.5 * t * torch.erfc(-t / math.sqrt(2)), "silu": lambda t: t * torch.sigmoid(t)}[activation](z)
    if activation != "none":
        error = 1.13 * error + y.abs() * 2.0 ** -20 + (2.0 ** -20 if activation == "gelu" else 0.0)
    if mul is not None:
        y, error = y * wide(mul), error * wide(mul).abs() + (y * wide(mul)).abs() * 2.0 ** -23
    if residual is not None:
        y = y + wide(residual)
        error = error + y.abs() * 2.0 ** -23
    return y, error


def kept(logits, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(tokens in the order in which a row draws, their weights) of one row of numbers; none: no token."""
    row = np.asarray(logits, dtype=np.float64)
    if not temperature >= 0 or np.isnan(row).any() or not (row > -np.inf).any():
        return [], []
    order = np.lexsort((np.arange(len(row)), -row))
    order = order[row[order] > -np.inf]
    top = row[order[0]]
    if temperature == 0 or top_k == 1:
        return order[:1], np.ones(1)
    if top == np.inf:
        order = order[row[order] == np.inf]
        w = np.ones(len(order))
    else:
        with np.errstate(over="ignore"):
            w = np.exp(-((top - row[order]) / np.float64(temperature)))
    if top_k > 0:
        order, w = order[:top_k], w[:top_k]
    n = len(w)
    if top_p < 1:
        n = min(n, int(np.searchsorted(np.cumsum(w), top_p * w.sum())) + 1)
    if min_p > 0:
        n = min(n, int((w >= min(min_p, 1.0)).sum()))
    return order[:n], w[:n]


def drawn(order, w, u):
    """(token, chance)"""
    if not len(order):
        return -1, 0.0
    upto = np.cumsum(w)
    at = min(int(np.searchsorted(upto, max(float(u), 0.0) * upto[-1], side="right")), len(w) - 1)
    return int(order[at]), float(w[at] / upto[-1])
