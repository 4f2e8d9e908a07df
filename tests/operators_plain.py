"""The operators beside the decoded weights, plainly and in 64 bits (on the CPU), with bounds of the error that 32-bit sums may have.  Shares no
code with the library."""
import math

import numpy as np
import torch

HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def wide(t):
    return t.detach().cpu().to(torch.float64)


def assert_within(got, want, bound, what=""):
    """|got - want| <= bound wherever want is finite; infinities and NaN in the same places."""
    got = wide(got)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), what
    off = ((got - want).abs() - bound)[fine]
    assert off.numel() == 0 or off.max().item() <= 0, (what, off.max().item(), int((off > 0).sum()))


def rms_norm(x, weight, eps, residual):
    """(y, h) in 64 bits."""
    h = wide(x) if residual is None else wide(x) + wide(residual)
    return h / torch.sqrt((h * h).mean(-1, keepdim=True) + eps) * wide(weight), h


def linear(x, w, x_scales=None, zero_point=0, scale=1.0, channel_scales=None, bias=None, activation="none", mul=None, residual=None):
    """(y, error): the product with its epilogue, and what sums of 32 bits may be off by: each of the k additions of a product of bf16
    numbers rounds once (8-bit sums are exact), scales and bias a few times, and no activation is steeper than 1.13."""
    a, b = wide(x), wide(w) - zero_point
    rows_by = wide(x_scales)[:, None] if x_scales is not None else torch.ones(a.shape[0], 1, dtype=torch.float64)
    cols_by = wide(channel_scales)[None] if channel_scales is not None else torch.ones(1, b.shape[0], dtype=torch.float64)
    by = rows_by * cols_by * scale
    y = a @ b.T * by
    size = a.abs() @ b.abs().T * by.abs()
    error = size * 2.0 ** -24 * (a.shape[1] if x.dtype == torch.bfloat16 else 0) + y.abs() * 2.0 ** -21
    if bias is not None:
        y = y + wide(bias)
        error = error + y.abs() * 2.0 ** -23
    y = {"none": lambda t: t, "relu": torch.relu, "gelu": lambda t: 0.5 * t * torch.erfc(-t / math.sqrt(2)), "silu": lambda t: t * torch.sigmoid(t)}[activation](y)
    if activation != "none":
        # erf and exp of 32 bits; gelu's 1 + erf loses what is below 2^-23 of 1
        error = 1.13 * error + y.abs() * 2.0 ** -20 + (2.0 ** -20 if activation == "gelu" else 0.0)
    if mul is not None:
        y, error = y * wide(mul), error * wide(mul).abs() + y.abs() * wide(mul).abs() * 2.0 ** -23
    if residual is not None:
        y = y + wide(residual)
        error = error + y.abs() * 2.0 ** -23
    return y, error


def quantise(x, bits):
    """(symbols, scales, zero-points) of vectors in the last dimension: every operation is one of 32 bits."""
    x = x.detach().cpu().to(torch.float32).numpy()
    most = np.float32((1 << bits) - 1)
    lo, hi = np.minimum(x.min(-1), np.float32(0)), np.maximum(x.max(-1), np.float32(0))
    with np.errstate(all="ignore"):
        scale = ((hi - lo) * (np.float32(1) / most)).astype(np.float32)
        fine = np.isfinite(x).all(-1) & np.isfinite(scale)
        by = np.where(fine & (scale > 0), scale, np.float32(1))
        zero = np.where(fine & (scale > 0), np.rint(-lo / by), np.float32(0)).astype(np.float32)
        q = np.rint(x / by[..., None]) + zero[..., None]
    q = np.where((fine & (scale > 0))[..., None], np.clip(q, 0, most), 0).astype(np.uint8)
    return q, np.where(fine, scale, np.float32(np.nan)), zero


def packed(q, bits):
    return q if bits == 8 else (q[..., 0::2] | (q[..., 1::2] << 4)).astype(np.uint8)


def values(symbols, params, bits):
    """fp64 values of a cache's arrays [..., D * bits / 8] and [..., 2]."""
    q = symbols.cpu().numpy()
    if bits == 4:
        q = np.stack([q & 15, q >> 4], axis=-1).reshape(*q.shape[:-1], -1)
    w = params.cpu().numpy().astype(np.float64)
    return torch.from_numpy((q.astype(np.float64) - w[..., 1:]) * w[..., :1])


def attend(q, k, v, tables, lengths, starts, page_size, scale):
    """(out, error): k, v the cache's values [pages, heads, page, D]; a page outside the cache is not seen.  Weights are rounded to 11 bits (two
    roundings with the scale's), scores are sums of D products in 32 bits, whose error is the weights' relative error."""
    q = wide(q)
    pages, heads, _, d = k.shape
    group = q.shape[1] // heads
    out, error = torch.zeros_like(q), torch.zeros_like(q)
    for s in range(len(lengths)):
        length, a, b = int(lengths[s]), int(starts[s]), int(starts[s + 1])
        at = torch.arange(length)
        page = tables[s].long().cpu()[at // page_size]
        held = (page >= 0) & (page < pages)
        page = torch.where(held, page, 0)
        for h in range(heads):
            kk, vv = k[page, h, at % page_size], v[page, h, at % page_size]
            for i in range(b - a):
                see = held & (at <= length - (b - a) + i)
                if not see.any():
                    continue
                for m in range(h * group, (h + 1) * group):
                    one = q[a + i, m]
                    scores = kk[see] @ one * scale
                    p = torch.softmax(scores, 0)
                    out[a + i, m] = p @ vv[see]
                    off = (kk[see].abs() @ one.abs() * abs(scale)).max() * 2.0 ** -24 * (d + 8) if torch.isfinite(scores).all() else 0.0
                    error[a + i, m] = (p @ vv[see].abs()) * (2.0 ** -10 + 4 * off) + vv[see].abs().max(0).values * 2.0 ** -26
    return out, error
