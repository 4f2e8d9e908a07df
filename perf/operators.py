"""What is measured of the operators that run a stack of compressed linear layers as a model: the norm with 8-bit output,
the product with its epilogue, the quantised cache and the attention that reads it.

A program that decodes the block of a 4096 / 11008 linear stack (4 matrices of 4096 x 4096, 3 of 4096 x 11008) to symbols or to
bf16 goes on with these: it adds the residual and normalises, multiplies, writes keys and values to a paged cache in 8 or
4 bits and attends over it.  32 heads of 128 make up 4096; fewer heads of keys and values than of queries, other widths and odd sizes
are drawn.  `own` false: plain torch in 32 bits, rounded once at the end; true: the library's calls.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


def listed():
    return [
        # the norm of one token's hidden state: launch and latency
        {"name": "norm_one_token", "kind": "norm", "rows": 1, "cols": 4096, "dtype": "bf16", "residual": True, "out": "bf16"},
        # the norm before a product in 8 bits, over a prompt
        {"name": "norm_prompt_8", "kind": "norm", "rows": 4096, "cols": 4096, "dtype": "bf16", "residual": True, "out": "i8"},
        # one token through the gate matrix of the stack, in 8 bits, times the other branch: the symbols are read once
        {"name": "linear_one_token_8", "kind": "linear", "rows": 1, "cols": 11008, "k": 4096, "x": "i8", "zero_point": 8, "bits": 4,
         "bias": False, "activation": "silu", "mul": True, "residual": False, "out": "bf16"},
        # sixteen sequences that take a token each through the matrix back to 4096, weights decoded to bf16
        {"name": "linear_few_tokens", "kind": "linear", "rows": 16, "cols": 4096, "k": 11008, "x": "bf16", "zero_point": 0, "bits": 0,
         "bias": False, "activation": "none", "mul": False, "residual": True, "out": "bf16"},
        # a ragged prompt, bf16 weights, bias and residual
        {"name": "linear_prompt", "kind": "linear", "rows": 3001, "cols": 4096, "k": 4096, "x": "bf16", "zero_point": 0, "bits": 0,
         "bias": True, "activation": "gelu", "mul": False, "residual": True, "out": "bf16"},
        # several prompts at once through the gate matrix in 8 bits
        {"name": "linear_prompts_8", "kind": "linear", "rows": 8192, "cols": 11008, "k": 4096, "x": "i8", "zero_point": 8, "bits": 4,
         "bias": False, "activation": "silu", "mul": True, "residual": False, "out": "bf16"},
        # one decoding step of sixteen sequences: their new keys and values written and read
        {"name": "cache_step_8", "kind": "cache", "tokens": 16, "heads": 32, "dim": 128, "page": 16, "bits": 8, "dtype": "bf16"},
        # a long prompt written in 4 bits and read back
        {"name": "cache_prompt_4", "kind": "cache", "tokens": 8191, "heads": 32, "dim": 128, "page": 64, "bits": 4, "dtype": "bf16"},
        # one decoding step of one sequence with a long context, keys and values shared by four heads of queries each
        {"name": "attend_long_context", "kind": "attend", "seqs": 1, "new": 1, "length": 65000, "least": 65000, "heads": 8, "group": 4, "dim": 128,
         "page": 64, "bits": 8},
        # one decoding step of many sequences of all lengths, every head with its own keys and values, 4 bits
        {"name": "attend_step_4", "kind": "attend", "seqs": 48, "new": 1, "length": 4100, "least": 17, "heads": 32, "group": 1, "dim": 128,
         "page": 16, "bits": 4},
        # chunks of prompts after what the cache holds already
        {"name": "attend_chunk", "kind": "attend", "seqs": 3, "new": 1531, "length": 6007, "least": 1531, "heads": 8, "group": 4, "dim": 128,
         "page": 64, "bits": 8},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A model's width: mostly a multiple of 64, sometimes any number."""
    n = _log_int(rng, lo, hi)
    return n if rng.random() < 0.25 else max(64, n // 64 * 64)


def draw(rng):
    kind = rng.choice(("norm", "linear", "linear", "linear", "cache", "attend", "attend", "attend"))
    if kind == "norm":
        cols = _width(rng, 64, 11008)
        return {"kind": kind, "rows": _log_int(rng, 1, min(16384, (1 << 25) // cols)), "cols": cols, "dtype": rng.choice(("bf16", "bf16", "f32")),
                "residual": rng.random() < 0.7, "out": rng.choice(("bf16", "i8"))}
    if kind == "linear":
        k, cols = _width(rng, 64, 11008), _width(rng, 64, 11008)
        x = rng.choice(("bf16", "i8"))
        rows = rng.randint(1, 32) if rng.random() < 0.4 else _log_int(rng, 1, 8192)
        bits = rng.choice((2, 4, 4, 6, 8)) if x == "i8" else 0
        return {"kind": kind, "rows": rows, "cols": cols, "k": k, "x": x, "zero_point": 0 if not bits else rng.choice((1 << (bits - 1), rng.randint(0, (1 << bits) - 1))),
                "bits": bits, "bias": rng.random() < 0.5, "activation": rng.choice(("none", "relu", "gelu", "silu")), "mul": rng.random() < 0.3,
                "residual": rng.random() < 0.5, "out": rng.choice(("bf16", "bf16", "f32"))}
    heads, dim = rng.choice((1, 2, 4, 8, 8, 16, 32)), rng.choice((64, 128, 128, 256))
    page, bits = rng.choice((16, 32, 64, 256)), rng.choice((8, 8, 4))
    if kind == "cache":
        return {"kind": kind, "tokens": _log_int(rng, 1, min(32768, (1 << 25) // (heads * dim))), "heads": heads, "dim": dim, "page": page, "bits": bits,
                "dtype": rng.choice(("bf16", "bf16", "f32"))}
    group = rng.choice((1, 1, 4, 8, rng.randint(2, 16)))
    group = min(group, 32 // heads)
    new = 1 if rng.random() < 0.5 else _log_int(rng, 2, 1531)
    # at most as many scores as the listed chunks have, and a cache of at most 2^28 elements each
    seqs = _log_int(rng, 1, 48 if new == 1 else 8)
    length = _log_int(rng, max(new, 16), 65000)
    most = min((1 << 28) // (seqs * heads * dim), int(8.8e8 * 128 / dim) // (seqs * heads * group * new))
    length = max(new, min(length, most))
    if length * new * seqs * heads * group * dim > 8.8e8 * 128:
        seqs = max(1, int(8.8e8 * 128 / (length * new * heads * group * dim)))
    return {"kind": kind, "seqs": seqs, "new": new, "length": length, "least": rng.randint(new, length), "heads": heads, "group": group, "dim": dim,
            "page": page, "bits": bits}


# ------------------------------------------------------------------------------------------------ inputs
def _lengths(case):
    """The sequences' lengths, new tokens included: from the least to the longest."""
    n, a, b = case["seqs"], case["least"], case["length"]
    return [b if n == 1 else a + (b - a) * i // (n - 1) for i in range(n)]


def _new_counts(case):
    """The new tokens of each sequence: the last ones have fewer than the first."""
    return [max(1, case["new"] - (case["new"] - 1) * i // (2 * case["seqs"])) for i in range(case["seqs"])]


def _filled_cache(case, total_pages, g):
    """Symbols and (scale, zero-point) pairs [pages, heads, page, ...] of keys and values that were written before."""
    h, p, d, bits = case["heads"], case["page"], case["dim"], case["bits"]
    most = (1 << bits) - 1
    out = []
    for _ in range(2):
        q = (torch.randn(total_pages, h, p, d, device=DEV, generator=g) * (most / 7.0) + most / 2.0).round_().clamp_(0, most).to(torch.uint8)
        if bits == 4:
            q = q[..., 0::2] | (q[..., 1::2] << 4)
        scale = (torch.rand(total_pages, h, p, 1, device=DEV, generator=g) + 0.5) * (7.0 / most)
        zero = torch.randint(int(0.4 * most), int(0.6 * most) + 1, (total_pages, h, p, 1), device=DEV, generator=g).float()
        out.append((q.contiguous(), torch.cat([scale, zero], dim=-1).contiguous()))
    return out


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    rnd = lambda *shape: torch.randn(*shape, device=DEV, generator=g)  # noqa: E731
    s = {"case": case}
    if case["kind"] == "norm":
        dt = TORCH[case["dtype"]]
        # hidden states have a few channels that are much larger than the others
        loud = 1.0 + 8.0 * (torch.rand(case["cols"], device=DEV, generator=g) < 0.01).float()
        s["x"] = (rnd(case["rows"], case["cols"]) * loud).to(dt)
        s["residual"] = (rnd(case["rows"], case["cols"]) * 2.0 * loud).to(dt) if case["residual"] else None
        s["weight"] = (1.0 + 0.2 * rnd(case["cols"])).to(dt)
    elif case["kind"] == "linear":
        r, c, k = case["rows"], case["cols"], case["k"]
        if case["x"] == "i8":
            s["x"] = (rnd(r, k) * 32.0).round_().clamp_(-127, 127).to(torch.int8)
            s["x_scales"] = (torch.rand(r, device=DEV, generator=g) + 0.5) / 32.0
            most = (1 << case["bits"]) - 1
            s["weight"] = (rnd(c, k) * ((most + 1) / 8.0) + case["zero_point"]).round_().clamp_(0, most).to(torch.uint8)
            s["scales"] = (torch.rand(c, device=DEV, generator=g) + 0.5) * (8.0 / ((most + 1) * math.sqrt(k)))
        else:
            s["x"] = rnd(r, k).to(torch.bfloat16)
            s["weight"] = (rnd(c, k) / math.sqrt(k)).to(torch.bfloat16)
        dt = TORCH[case["out"]]
        s["bias"] = 0.1 * rnd(c) if case["bias"] else None
        s["mul"] = rnd(r, c).to(dt) if case["mul"] else None
        s["residual"] = rnd(r, c).to(dt) if case["residual"] else None
    elif case["kind"] == "cache":
        n, h, d, p = case["tokens"], case["heads"], case["dim"], case["page"]
        # keys and values are slices of what one product gave for queries, keys and values
        qkv = rnd(n, 3 * h * d).to(TORCH[case["dtype"]]).view(n, 3, h, d)
        s["k"], s["v"] = qkv[:, 1], qkv[:, 2]
        pages = -(-n // p) + 3
        s["cache"] = [(torch.zeros(pages, h, p, d * case["bits"] // 8, dtype=torch.uint8, device=DEV), torch.zeros(pages, h, p, 2, device=DEV)) for _ in range(2)]
        order = torch.randperm(pages, device=DEV, generator=g)[: -(-n // p)]
        s["slots"] = (order[:, None] * p + torch.arange(p, device=DEV)).reshape(-1)[:n].contiguous()
    else:
        lengths, news, h, d, p = _lengths(case), _new_counts(case), case["heads"], case["dim"], case["page"]
        counts = [-(-n // p) for n in lengths]
        total = sum(counts) + 2
        s["cache"] = _filled_cache(case, total, g)
        order = torch.randperm(total, device=DEV, generator=g).to(torch.int32)
        table, at = torch.zeros(len(lengths), max(counts), dtype=torch.int32, device=DEV), 0
        for i, n in enumerate(counts):
            table[i, :n] = order[at:at + n]
            at += n
        s["pages"] = table
        s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device=DEV)
        starts = [0]
        for n in news:
            starts.append(starts[-1] + n)
        s["starts"] = torch.tensor(starts, dtype=torch.int32, device=DEV)
        s["most_new"] = max(news)
        s["q"] = rnd(starts[-1], h * case["group"], d).to(torch.bfloat16)
    return s


# ------------------------------------------------------------------------------------------------ the operators
def run(s):
    case = s["case"]
    return (_OWN if own else _PLAIN)[case["kind"]](s, case)


def _binding():
    from paper_2406_06237_amd import binding
    return binding


def _own_norm(s, case):
    out, scales, total = _binding().rms_norm(s["x"], s["weight"], EPS, residual=s["residual"], out_dtype=case["out"])
    if case["out"] == "i8":
        out = _value_of_rows(out, scales)
    return [out] if total is None else [out, total]


def _own_linear(s, case):
    B = _binding()
    if case["x"] == "i8":
        return B.linear(s["x"], s["weight"], x_scales=s["x_scales"], zero_point=case["zero_point"], channel_scales=s["scales"], bias=s["bias"],
                        activation=case["activation"], mul=s["mul"], residual=s["residual"], out_dtype=case["out"])
    return B.linear(s["x"], s["weight"], bias=s["bias"], activation=case["activation"], mul=s["mul"], residual=s["residual"], out_dtype=case["out"])


def _own_handle(s, case):
    (k, kp), (v, vp) = s["cache"]
    return _binding().KvCache(k, kp, v, vp, case["bits"])


def _own_cache(s, case):
    B, cache = _binding(), _own_handle(s, case)
    B.cache_write(cache, s["k"], s["v"], s["slots"])
    return list(B.cache_read(cache, s["slots"], out_dtype="bf16"))


def _own_attend(s, case):
    return _binding().attend(s["q"], _own_handle(s, case), s["pages"], s["lengths"], s["starts"])


def _value_of_rows(q, scales):
    """8-bit rows as the values they stand for."""
    out = torch.empty(q.shape, dtype=torch.bfloat16, device=q.device)
    return torch.mul(q, scales[:, None], out=out)


def _plain_norm(s, case):
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    y = h * torch.rsqrt((h * h).mean(dim=-1, keepdim=True) + EPS) * s["weight"].float()
    if case["out"] == "i8":
        scales = y.abs().amax(dim=-1) / 127.0
        out = _value_of_rows(torch.round(y / scales[:, None].clamp_min(1e-38)).to(torch.int8), scales)
    else:
        out = y.to(TORCH[case["out"]])
    return [out] if s["residual"] is None else [out, h.to(s["x"].dtype)]


def _plain_linear(s, case):
    w = s["weight"].float()
    if case["x"] == "i8":
        w = (w - case["zero_point"]) * s["scales"][:, None]
    y = s["x"].float() @ w.t()
    if case["x"] == "i8":
        y = y * s["x_scales"][:, None]
    if s["bias"] is not None:
        y = y + s["bias"]
    if case["activation"] == "relu":
        y = torch.clamp_min(y, 0.0)
    elif case["activation"] == "gelu":
        y = 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5)))
    elif case["activation"] == "silu":
        y = y / (1.0 + torch.exp(-y))
    if s["mul"] is not None:
        y = y * s["mul"].float()
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(TORCH[case["out"]])


def _plain_quantised(x, bits):
    """Symbols and (scale, zero-point) of vectors in the last dimension."""
    most = (1 << bits) - 1
    x = x.float()
    lo, hi = x.amin(dim=-1, keepdim=True).clamp_max(0.0), x.amax(dim=-1, keepdim=True).clamp_min(0.0)
    scale = (hi - lo) / most
    safe = torch.where(scale > 0, scale, 1.0)
    zero = torch.round(-lo / safe)
    q = (torch.round(x / safe) + zero).clamp(0, most).to(torch.uint8)
    if bits == 4:
        q = q[..., 0::2] | (q[..., 1::2] << 4)
    return q, torch.cat([scale, zero], dim=-1)


def _plain_values(q, params, bits):
    if bits == 4:
        q = torch.stack([q & 15, q >> 4], dim=-1).flatten(-2)
    return (q.float() - params[..., 1:]) * params[..., :1]


def _plain_cache(s, case):
    p, out = case["page"], []
    page, at = s["slots"] // p, s["slots"] % p
    for x, (store, params) in zip((s["k"], s["v"]), s["cache"]):
        q, w = _plain_quantised(x, case["bits"])
        store[page, :, at] = q
        params[page, :, at] = w
        out.append(_plain_values(store[page, :, at], params[page, :, at], case["bits"]).to(torch.bfloat16))
    return out


def _plain_attend(s, case):
    h, d, n, group = case["heads"], case["dim"], case["seqs"], case["group"]
    kv = []
    for store, params in s["cache"]:
        x = _plain_values(store[s["pages"]], params[s["pages"]], case["bits"])          # [seqs, pages, heads, page, dim]
        kv.append(x.transpose(1, 2).reshape(n, h, -1, d))
    k, v = kv
    most, news = s["most_new"], (s["starts"][1:] - s["starts"][:-1]).long()
    i = torch.arange(most, device=DEV)
    there = i < news[:, None]                                                             # [seqs, most]
    rows = (s["starts"][:-1, None].long() + i).clamp_max(s["q"].shape[0] - 1)
    q = s["q"].float()[rows].view(n, most, h, group, d).permute(0, 2, 1, 3, 4).reshape(n, h, most * group, d)
    scores = q @ k.transpose(-1, -2).contiguous() * (1.0 / math.sqrt(d))
    last = s["lengths"].long()[:, None] - news[:, None] + i                               # the position of each new token
    seen = torch.arange(k.shape[2], device=DEV) <= last[:, :, None]                       # [seqs, most, positions]
    seen = seen[:, None, :, None, :].expand(n, h, most, group, -1).reshape(n, h, most * group, -1)
    scores = torch.where(seen, scores, -math.inf)
    top = scores.amax(dim=-1, keepdim=True)
    e = torch.exp(scores - torch.where(top == -math.inf, 0.0, top))
    o = (e @ v) / e.sum(dim=-1, keepdim=True).clamp_min(1e-38)
    o = o.view(n, h, most, group, d).permute(0, 2, 1, 3, 4).reshape(n, most, h * group, d)
    return o[there].to(torch.bfloat16)


_PLAIN = {"norm": _plain_norm, "linear": _plain_linear, "cache": _plain_cache, "attend": _plain_attend}
_OWN = {"norm": _own_norm, "linear": _own_linear, "cache": _own_cache, "attend": _own_attend}


# ------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    f64 = lambda t: t.to(torch.float64)  # noqa: E731
    if case["kind"] == "norm":
        total = f64(s["x"]) if s["residual"] is None else f64(s["x"]).add_(f64(s["residual"]))
        y = total / (total.pow(2).sum(1, keepdim=True) / case["cols"] + EPS).sqrt() * f64(s["weight"])
        if case["out"] == "i8":
            step = torch.linalg.vector_norm(y, ord=math.inf, dim=1, keepdim=True) / 127
            y = torch.round(y / step) * step
        return [y] if s["residual"] is None else [y, total]
    if case["kind"] == "linear":
        z = torch.mm(f64(s["x"]), (f64(s["weight"]) - case["zero_point"]).T)
        if case["x"] == "i8":
            z *= torch.outer(f64(s["x_scales"]), f64(s["scales"]))
        if s["bias"] is not None:
            z += f64(s["bias"])
        z = {"none": lambda t: t, "relu": torch.relu, "silu": lambda t: t * torch.sigmoid(t),
             "gelu": lambda t: 0.5 * t * torch.erfc(-t / math.sqrt(2))}[case["activation"]](z)
        if s["mul"] is not None:
            z *= f64(s["mul"])
        return z if s["residual"] is None else z + f64(s["residual"])
    if case["kind"] == "cache":
        # scale and quotients are numbers of 32 bits by definition; everything else is in 64
        out, most = [], 2 ** case["bits"] - 1
        for x in (s["k"], s["v"]):
            x = x.to(torch.float32).contiguous()
            low, high = torch.clamp(x.min(2).values, max=0), torch.clamp(x.max(2).values, min=0)
            step = ((high - low) / most)[..., None]
            zero = f64(torch.round(-low[..., None] / step))
            out.append(f64(step) * (torch.clamp(f64(torch.round(x / step)) + zero, 0, most) - zero))
        return out
    h, d, group, p = case["heads"], case["dim"], case["group"], case["page"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    at = 0
    for i, (length, new) in enumerate(zip(_lengths(case), _new_counts(case))):
        where = torch.arange(length, device=DEV)
        page, inside = s["pages"][i].long()[where // p], where % p
        hidden = where[None, :] > length - new + torch.arange(new, device=DEV)[:, None]
        for j in range(h):
            k, v = [], []
            for (store, params), to in zip(s["cache"], (k, v)):
                q = store[page, j, inside].long()
                if case["bits"] == 4:
                    both = torch.empty(length, d, dtype=torch.long, device=DEV)
                    both[:, ::2], both[:, 1::2] = q % 16, torch.div(q, 16, rounding_mode="floor")
                    q = both
                w = f64(params[page, j, inside])
                to.append(w[:, :1] * (q - w[:, 1:]))
            for m in range(j * group, (j + 1) * group):
                z = torch.mm(f64(s["q"][at:at + new, m]), k[0].T) / math.sqrt(d)
                out[at:at + new, m] = torch.mm(torch.softmax(z.masked_fill(hidden, -math.inf), dim=1), v[0])
        at += new
    return out


def work(case):
    if case["kind"] == "norm":
        n, size = case["rows"] * case["cols"], 4 if case["dtype"] == "f32" else 2
        moved = n * size * (3 if case["residual"] else 1) + n * (1 if case["out"] == "i8" else 2) + case["cols"] * size
        return {"bytes": moved, "flops": 6 * n}
    if case["kind"] == "linear":
        r, c, k = case["rows"], case["cols"], case["k"]
        size = 1 if case["x"] == "i8" else 2
        out = (4 if case["out"] == "f32" else 2) * r * c
        return {"bytes": size * (r * k + c * k) + 4 * c + out * (1 + case["mul"] + case["residual"]), "flops": 2 * r * c * k}
    h, d, each = case["heads"], case["dim"], case["dim"] * case["bits"] // 8 + 8
    if case["kind"] == "cache":
        n = 2 * case["tokens"] * h
        return {"bytes": n * (d * (4 if case["dtype"] == "f32" else 2) + 2 * each + 2 * d), "flops": 4 * n * d}
    lengths, news = _lengths(case), _new_counts(case)
    seen = sum(new * length - new * (new - 1) // 2 for length, new in zip(lengths, news))
    return {"bytes": 2 * h * each * sum(lengths) + 4 * sum(news) * h * case["group"] * d, "flops": 4 * seen * h * case["group"] * d}


if __name__ == "__main__":
    for c in listed() + [draw(random.Random(i)) for i in range(6)]:
        print(c, work(c))
