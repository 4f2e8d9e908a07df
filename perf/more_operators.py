"""What is measured of the operators that make a serving step of the block of compressed linear layers: tokens placed in the paged cache,
looked up as rows, low-rank adapters of many requests beside the block's products, and the next token drawn from the logits.

`own` false: plain torch in 32 bits (64 where values next to a border decide), rounded once at the end; true: the library's calls.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "i8": torch.int8, "u8": torch.uint8}


def listed():
    return [
        # one decoding step of sixteen sequences: a slot for each of their new tokens
        {"name": "place_step", "kind": "place", "seqs": 16, "page": 64, "held": 4000, "new": 1, "ends": 0, "spare": 40, "padding": 0},
        # a large batch: a quarter of the sequences end, most of the others take prompts of all lengths
        {"name": "place_prompts", "kind": "place", "seqs": 512, "page": 16, "held": 8000, "new": 4000, "ends": 4, "spare": 500, "padding": 133},
        # the rows of one decoding step's tokens, from decoded symbols
        {"name": "embed_step", "kind": "embed", "tokens": 16, "vocabulary": 32000, "cols": 4096, "weight": "u8", "zero_point": 8, "bits": 4, "out": "bf16"},
        # several prompts at once
        {"name": "embed_prompts", "kind": "embed", "tokens": 16384, "vocabulary": 65536, "cols": 4096, "weight": "u8", "zero_point": 131, "bits": 8, "out": "bf16"},
        # one request with its adapter: latency
        {"name": "adapt_one", "kind": "adapt", "rows": 1, "seqs": 1, "k": 4096, "cols": 4096, "rank": 16, "adapters": 8, "without": False, "x": "i8", "base": "bf16",
         "out": "bf16", "activation": "none", "mul": False, "residual": True},
        # one decoding step of 64 requests that have 48 adapters among them, at the gate
        {"name": "adapt_step", "kind": "adapt", "rows": 64, "seqs": 64, "k": 4096, "cols": 11008, "rank": 16, "adapters": 48, "without": True, "x": "i8", "base": "bf16",
         "out": "bf16", "activation": "silu", "mul": False, "residual": False},
        # a chunk of two prompts and some single tokens, the matrix back to 4096, rank no power of two
        {"name": "adapt_chunk", "kind": "adapt", "rows": 1531, "seqs": 9, "k": 11008, "cols": 4096, "rank": 24, "adapters": 5, "without": True, "x": "bf16",
         "base": "f32", "out": "f32", "activation": "none", "mul": False, "residual": True},
        # several prompts at the gate, times the other branch
        {"name": "adapt_prompts", "kind": "adapt", "rows": 8192, "seqs": 16, "k": 4096, "cols": 11008, "rank": 64, "adapters": 8, "without": False, "x": "i8",
         "base": "bf16", "out": "bf16", "activation": "silu", "mul": True, "residual": False},
        # the next token of one request: latency
        {"name": "sample_one", "kind": "sample", "rows": 1, "vocabulary": 32000, "dtype": "f32", "top_k": 0, "top_p": 0.9, "min_p": 0.0, "greedy": 0, "masked": 0.0},
        # 64 requests, each with settings of its own
        {"name": "sample_step", "kind": "sample", "rows": 64, "vocabulary": 131072, "dtype": "f32", "top_k": 50, "top_p": 0.95, "min_p": 0.05, "greedy": 8, "masked": 0.0},
        # an odd vocabulary of which a grammar leaves a part, nothing else cut off
        {"name": "sample_grammar", "kind": "sample", "rows": 48, "vocabulary": 50001, "dtype": "bf16", "top_k": 0, "top_p": 1.0, "min_p": 0.0, "greedy": 0, "masked": 0.7},
        # many samples of few prompts, by probability alone
        {"name": "sample_many", "kind": "sample", "rows": 512, "vocabulary": 131072, "dtype": "bf16", "top_k": 0, "top_p": 0.9, "min_p": 0.02, "greedy": 0, "masked": 0.0},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A model's width: mostly a multiple of 64, sometimes any number."""
    n = _log_int(rng, lo, hi)
    return n if rng.random() < 0.25 else max(64, n // 64 * 64)


def draw(rng):
    kind = rng.choice(("place", "embed", "adapt", "adapt", "adapt", "sample", "sample", "sample"))
    if kind == "place":
        seqs = _log_int(rng, 1, 512)
        new = 1 if rng.random() < 0.5 else _log_int(rng, 2, 4000)
        return {"kind": kind, "seqs": seqs, "page": rng.choice((16, 16, 32, 64, 256)), "held": _log_int(rng, 16, 8000), "new": new, "ends": rng.choice((0, 0, 3, 4, 9)),
                # (fewer pages than are asked for: the last sequences are refused)
                "spare": rng.choice((rng.randint(0, 500), rng.randint(0, 500), -rng.randint(1, 9))), "padding": rng.choice((0, rng.randint(1, 200)))}
    if kind == "embed":
        cols, bits = _width(rng, 64, 11008), rng.choice((2, 4, 6, 8))
        return {"kind": kind, "tokens": _log_int(rng, 1, min(16384, (1 << 26) // cols)), "vocabulary": _log_int(rng, 1000, min(131072, (1 << 28) // cols)), "cols": cols,
                "weight": rng.choice(("u8", "u8", "bf16")), "zero_point": rng.randint(0, (1 << bits) - 1), "bits": bits, "out": rng.choice(("bf16", "bf16", "f32"))}
    if kind == "adapt":
        k, cols = _width(rng, 64, 11008), _width(rng, 64, 11008)
        rows = rng.randint(1, 64) if rng.random() < 0.5 else _log_int(rng, 1, 8192)
        rank = rng.choice((4, 8, 16, 16, 32, 64, 128, rng.randint(1, 100)))
        adapters = _log_int(rng, 1, 64)
        # at most as many multiplications and bytes as the listed prompts at the gate
        adapters = max(1, min(adapters, 512 * 8192 // (rows * rank)))
        rows = max(1, min(rows, 512 * 8192 // (rank * adapters)))
        case = {"kind": kind, "rows": rows, "seqs": 1, "k": k, "cols": cols, "rank": rank, "adapters": adapters,
                "without": rng.random() < 0.4, "x": rng.choice(("bf16", "i8", "i8")), "base": rng.choice(("bf16", "bf16", "f32")), "out": rng.choice(("bf16", "bf16", "f32")),
                "activation": rng.choice(("none", "none", "relu", "gelu", "silu")), "mul": rng.random() < 0.2, "residual": rng.random() < 0.4}
        most = work(next(c for c in listed() if c["name"] == "adapt_prompts"))
        while any(work(case)[what] > most[what] for what in most):
            case["rows"] = case["rows"] * 3 // 4
        case["seqs"] = case["rows"] if rng.random() < 0.4 else rng.randint(1, min(case["rows"], 32))
        return case
    vocabulary = _log_int(rng, 1000, 131072)
    top_p = rng.choice((1.0, 0.9, 0.5, round(rng.uniform(0.1, 0.99), 2)))
    return {"kind": kind, "rows": rng.randint(1, 64) if rng.random() < 0.6 else _log_int(rng, 1, 512), "vocabulary": vocabulary, "dtype": rng.choice(("f32", "f32", "bf16")),
            "top_k": rng.choice((0, 0, 1, 20, 50, rng.randint(2, 1000))), "top_p": top_p, "min_p": rng.choice((0.0, 0.0, 0.05, round(rng.uniform(0.001, 0.3), 3))),
            "greedy": rng.choice((0, 0, 3, 8)), "masked": rng.choice((0.0, 0.0, 0.5, 0.9))}


# ------------------------------------------------------------------------------------------------ inputs
def _held(case):
    """Tokens that the sequences hold, and how many each is to get; what a seed changes is which sequence has which."""
    n = case["seqs"]
    held = [case["held"] * (3 * i % n + 1) // n for i in range(n)]
    if case["new"] == 1:
        new = [1] * n
    else:
        new = [int(round(case["new"] ** ((7 * i % n + 1) / n))) if i % 5 else 1 for i in range(n)]
    # (a sequence that ends gets nothing in the same step, so that the pages it gives back are still in its row when the step is done again)
    return held, [0 if _ended(case, i) else m for i, m in enumerate(new)]


def _ended(case, i):
    return bool(case["ends"]) and i % case["ends"] == 1


def _pages_of(case):
    """Pages held, pages asked for behind the ended sequences' return, and the table's width."""
    p, (held, new) = case["page"], _held(case)
    up = lambda n: -(-n // p)  # noqa: E731
    kept = [0 if _ended(case, i) else h for i, h in enumerate(held)]
    asked = sum(up(h + n) - up(h) for h, n in zip(kept, new))
    returned = sum(up(h) for h in held) - sum(up(h) for h in kept)
    return sum(up(h) for h in held), asked, returned, up(case["held"] + case["new"]) + 3


def _rows_of_sequences(case):
    """Rows of each sequence: single ones and long ones."""
    n, rows = case["seqs"], case["rows"]
    if n == rows:
        return [1] * n
    shares = [1 + (i * i) % 7 * 3 for i in range(n)]
    counts = [max(1, (rows - n) * s // sum(shares) + 1) for s in shares]
    counts[0] += rows - sum(counts)
    return counts


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    rnd = lambda *shape: torch.randn(*shape, device=DEV, generator=g)  # noqa: E731
    uniform = lambda *shape: torch.rand(*shape, device=DEV, generator=g)  # noqa: E731
    s = {"case": case}
    if case["kind"] == "place":
        n, p, (held, new) = case["seqs"], case["page"], _held(case)
        total, asked, returned, width = _pages_of(case)
        order = random.Random(seed).sample(range(n), n)
        ints = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
        held, ends = [held[i] for i in order], [int(_ended(case, i)) for i in order]
        s["lengths"], s["new"], s["ends"] = ints(held), ints([new[i] for i in order]), ints(ends) if case["ends"] else None
        there = max(0, asked - returned + case["spare"])
        deal = torch.randperm(total + there, device=DEV, generator=g).to(torch.int32)
        counts = torch.tensor([-(-h // p) for h in held], device=DEV)
        where = torch.arange(width, device=DEV) < counts[:, None]
        s["pages"] = torch.full((n, width), -1, dtype=torch.int32, device=DEV)
        s["pages"][where] = deal[:total]
        s["free"] = torch.zeros(total + there, dtype=torch.int32, device=DEV)
        s["free"][:there] = deal[total:]
        s["n_free"] = ints([there])
        s["n_tokens"] = sum(new) + case["padding"]
    elif case["kind"] == "embed":
        v, c = case["vocabulary"], case["cols"]
        if case["weight"] == "u8":
            s["weight"] = torch.randint(0, 1 << case["bits"], (v, c), dtype=torch.uint8, device=DEV, generator=g)
            s["row_scales"] = (uniform(v) + 0.5) * (4.0 / (1 << case["bits"]))
            s["scale"] = math.sqrt(c)
        else:
            s["weight"] = rnd(v, c).to(torch.bfloat16)
            s["row_scales"], s["scale"] = None, math.sqrt(c)
        # few tokens are frequent
        s["tokens"] = (uniform(case["tokens"]).double() ** 3 * v).long().clamp_(0, v - 1)
    elif case["kind"] == "adapt":
        r, k, c, rank, n = case["rows"], case["k"], case["cols"], case["rank"], case["adapters"]
        if case["x"] == "i8":
            s["x"] = (rnd(r, k) * 32.0).round_().clamp_(-127, 127).to(torch.int8)
            s["x_scales"] = (uniform(r) + 0.5) / 32.0
        else:
            s["x"], s["x_scales"] = rnd(r, k).to(torch.bfloat16), None
        s["a"] = (rnd(n, rank, k) / math.sqrt(k)).to(torch.bfloat16)
        s["b"] = (rnd(n, c, rank) / math.sqrt(rank)).to(torch.bfloat16)
        s["scales"] = uniform(n) + 0.5
        counts = torch.tensor(_rows_of_sequences(case), device=DEV)
        ids = torch.randint(-1 if case["without"] else 0, n, (case["seqs"],), dtype=torch.int32, device=DEV, generator=g)
        s["ids"] = torch.repeat_interleave(ids, counts, output_size=r)
        s["base"] = rnd(r, c).to(TORCH[case["base"]])
        s["mul"] = rnd(r, c).to(TORCH[case["out"]]) if case["mul"] else None
        s["residual"] = rnd(r, c).to(TORCH[case["out"]]) if case["residual"] else None
    else:
        r, v = case["rows"], case["vocabulary"]
        x = rnd(r, v) * 2.5
        # a few tokens stand out, more in some rows than in others
        x += (uniform(r, v) < 30.0 / v) * (uniform(r, 1) * 12.0)
        if case["masked"]:
            x = torch.where(uniform(r, v) < case["masked"], -math.inf, x)
        s["logits"] = x.to(TORCH[case["dtype"]])
        s["uniforms"] = uniform(r)
        temperature = uniform(r) * 0.7 + 0.6
        s["top_k"], s["top_p"], s["min_p"] = case["top_k"], case["top_p"], case["min_p"]
        if case["greedy"]:                                      # requests with settings of their own, some of them greedy
            temperature[::case["greedy"]] = 0.0
            s["top_k"] = torch.randint(0, 2 * case["top_k"] + 1, (r,), dtype=torch.int32, device=DEV, generator=g)
            s["top_p"] = 1.0 - (1.0 - case["top_p"]) * 2.0 * uniform(r).clamp_max(0.5)
            s["min_p"] = case["min_p"] * uniform(r)
        s["temperature"] = temperature
    return s


# ------------------------------------------------------------------------------------------------ the operators
def run(s):
    case = s["case"]
    return (_OWN if own else _PLAIN)[case["kind"]](s, case)


def _binding():
    from paper_2406_06237_amd import binding
    return binding


def _own_place(s, case):
    placed = _binding().place_tokens(s["pages"], case["page"], s["lengths"], s["new"], s["free"], s["n_free"], s["n_tokens"], ends=s["ends"])
    return [*placed, s["pages"], s["free"]]


def _own_embed(s, case):
    return _binding().embed(s["tokens"], s["weight"], zero_point=case["zero_point"] if case["weight"] == "u8" else 0, row_scales=s["row_scales"], scale=s["scale"],
                            out_dtype=case["out"])


def _own_adapt(s, case):
    return _binding().adapt(s["base"], s["x"], s["a"], s["b"], s["ids"], x_scales=s["x_scales"], scales=s["scales"], activation=case["activation"], mul=s["mul"],
                            residual=s["residual"], out_dtype=case["out"])


def _own_sample(s, case):
    # the tokens, and the probability with which each was drawn
    return _binding().sample(s["logits"], s["uniforms"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])


def _plain_place(s, case):
    p, pages, free, n_tokens = case["page"], s["pages"], s["free"], s["n_tokens"]
    width, capacity = pages.shape[1], free.shape[0]
    lengths, new = s["lengths"].long(), s["new"].long()
    ended = torch.zeros_like(lengths, dtype=torch.bool) if s["ends"] is None else s["ends"] != 0
    # the ended sequences' pages go back on the stack, sequence by sequence
    column = torch.arange(width, device=DEV)
    back = torch.where(ended, (lengths + p - 1) // p, 0)
    first = s["n_free"].long() + torch.cumsum(back, 0) - back
    to = torch.where(column < back[:, None], first[:, None] + column, capacity)
    stack = torch.cat([free, free.new_zeros(1)])
    stack[to.reshape(-1)] = pages.reshape(-1)
    free.copy_(stack[:capacity])
    top = s["n_free"].long() + back.sum()
    # what each sequence needs more, dealt in order from the stack's end
    old = torch.where(ended, 0, lengths)
    have, want = (old + p - 1) // p, (old + new + p - 1) // p
    need = want - have
    upto = torch.cumsum(need, 0)
    served = (need == 0) | (upto <= top)
    after = torch.where(served, old + new, old)
    taken = torch.where(served & (need > 0), upto, 0).amax()
    at = top - 1 - ((upto - need)[:, None] + column - have[:, None])
    dealt = (column >= have[:, None]) & (column < want[:, None]) & served[:, None]
    pages.copy_(torch.where(dealt, free[at.clamp(0, capacity - 1)], pages))
    # and where its new tokens go
    ends = torch.cumsum(new, 0)
    starts = torch.cat([ends.new_zeros(1), ends])
    t = torch.arange(n_tokens, device=DEV)
    owner = torch.searchsorted(ends, t, right=True)
    there = owner < lengths.shape[0]
    owner = owner.clamp_max(lengths.shape[0] - 1)
    position = old[owner] + t - starts[owner]
    good = there & served[owner]
    slot = pages[owner, (position // p).clamp(0, width - 1)].long() * p + position % p
    return [torch.where(good, slot, -1), starts.int(), after.int(), torch.where(there, owner, -1).int(), (top - taken).int(), pages, free]


def _plain_embed(s, case):
    rows = s["weight"][s["tokens"]].float()
    if case["weight"] == "u8":
        rows = (rows - case["zero_point"]) * s["row_scales"][s["tokens"]][:, None]
    return (rows * s["scale"]).to(TORCH[case["out"]])


def _plain_adapt(s, case):
    n, rank, c = case["adapters"], case["rank"], case["cols"]
    # all adapters side by side; a row keeps what its own one gives
    h = s["x"].float() @ s["a"].float().reshape(n * rank, -1).t()
    if s["x_scales"] is not None:
        h = h * s["x_scales"][:, None]
    mine = s["ids"][:, None] == torch.arange(n, device=DEV)
    h = torch.where(mine[:, :, None], h.view(-1, n, rank) * s["scales"][:, None], 0.0).view(-1, n * rank)
    y = s["base"].float() + h @ s["b"].float().permute(0, 2, 1).reshape(n * rank, c)
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


def _settings(s, case):
    """Temperature, top_k, top_p and min_p as columns of a number for each row."""
    r = case["rows"]
    column = lambda v, t: (v.to(t) if torch.is_tensor(v) else torch.full((r,), v, dtype=torch.float32, device=DEV).to(t))[:, None]  # noqa: E731
    return column(s["temperature"], torch.float64), column(s["top_k"], torch.int64), column(s["top_p"], torch.float64), column(s["min_p"], torch.float64)


def _plain_sample(s, case):
    temperature, top_k, top_p, min_p = _settings(s, case)
    x, index = torch.sort(s["logits"].float(), dim=-1, descending=True, stable=True)
    x = x.double()
    x = torch.where(x == -math.inf, -math.inf, (x - x[:, :1]) / torch.where(temperature > 0, temperature, 1.0))
    w = torch.exp(x)
    place = torch.arange(x.shape[1], device=DEV)
    w = torch.where((temperature > 0) | (place == 0), w, 0.0)
    w = torch.where((top_k == 0) | (place < top_k), w, 0.0)
    mass = torch.cumsum(w, dim=-1)
    w = torch.where((top_p >= 1.0) | (place == 0) | (mass - w < top_p * mass[:, -1:]), w, 0.0)
    w = torch.where(w >= min_p, w, 0.0)
    mass = torch.cumsum(w, dim=-1)
    at = (mass <= s["uniforms"].double()[:, None] * mass[:, -1:]).sum(dim=-1, keepdim=True)
    last = (w > 0).sum(dim=-1, keepdim=True) - 1
    at = torch.minimum(at, last)
    return [index.gather(1, at)[:, 0], (w.gather(1, at) / mass[:, -1:])[:, 0].float()]


_PLAIN = {"place": _plain_place, "embed": _plain_embed, "adapt": _plain_adapt, "sample": _plain_sample}
_OWN = {"place": _own_place, "embed": _own_embed, "adapt": _own_adapt, "sample": _own_sample}


# ------------------------------------------------------------------------------------------------ in 64 bits
def _exact_place(s, case):
    """One sequence behind the other, as a program on the host would."""
    p, n_tokens = case["page"], s["n_tokens"]
    table, free, n_free = s["pages"].tolist(), s["free"].tolist(), int(s["n_free"])
    lengths, new = s["lengths"].tolist(), s["new"].tolist()
    ends = [0] * len(lengths) if s["ends"] is None else s["ends"].tolist()
    stack = free[:n_free]
    for i, e in enumerate(ends):
        if e:
            stack += table[i][:math.ceil(lengths[i] / p)]
            lengths[i] = 0
    free[:len(stack)] = stack
    slots, owners, starts, short = [], [], [0], False
    for i, n in enumerate(new):
        more = math.ceil((lengths[i] + n) / p) - math.ceil(lengths[i] / p)
        short = short or more > len(stack)
        starts.append(starts[-1] + n)
        owners += [i] * n
        if short and more:
            slots += [-1] * n
            continue
        for j in range(n):
            at = lengths[i] + j
            if at % p == 0:
                table[i][at // p] = stack.pop()
            slots.append(table[i][at // p] * p + at % p)
        lengths[i] += n
    rest = [-1] * (n_tokens - len(slots))
    ints = lambda a, t=torch.int32: torch.tensor(a, dtype=t, device=DEV)  # noqa: E731
    return [ints(slots + rest, torch.int64), ints(starts), ints(lengths), ints(owners + rest), ints([len(stack)]), ints(table), ints(free)]


def exact(case, seed):
    s = prepare(case, seed)
    f64 = lambda t: t.to(torch.float64)  # noqa: E731
    if case["kind"] == "place":
        return _exact_place(s, case)
    if case["kind"] == "embed":
        picked = f64(torch.index_select(s["weight"], 0, s["tokens"]))
        by = torch.full((case["tokens"], 1), s["scale"], dtype=torch.float64, device=DEV)
        if case["weight"] == "u8":
            picked -= case["zero_point"]
            by = by * f64(torch.index_select(s["row_scales"], 0, s["tokens"]))[:, None]
        return picked * by
    if case["kind"] == "adapt":
        z = f64(s["base"])
        for i in range(case["adapters"]):
            rows = torch.nonzero(s["ids"] == i)[:, 0]
            if len(rows):
                inner = torch.mm(f64(s["x"][rows]), f64(s["a"][i]).T)
                if s["x_scales"] is not None:
                    inner *= f64(s["x_scales"][rows])[:, None]
                z[rows] += torch.mm(inner, f64(s["b"][i]).T) * f64(s["scales"][i])
        z = {"none": lambda t: t, "relu": torch.relu, "silu": lambda t: t * torch.sigmoid(t),
             "gelu": lambda t: 0.5 * t * torch.erfc(-t / math.sqrt(2))}[case["activation"]](z)
        if s["mul"] is not None:
            z *= f64(s["mul"])
        return z if s["residual"] is None else z + f64(s["residual"])
    # one row behind the other: a list of its tokens by falling logit, cut three times
    import numpy as np
    temperature, top_k, top_p, min_p = (t.reshape(-1).cpu().numpy() for t in _settings(s, case))
    logits, u = s["logits"].float().cpu().numpy(), f64(s["uniforms"]).cpu().numpy()
    tokens, chances = [], []
    for i, row in enumerate(logits):
        if temperature[i] == 0.0:
            tokens.append(int(np.argmax(row)))
            chances.append(1.0)
            continue
        order = np.lexsort((np.arange(len(row)), -row))
        order = order[row[order] > -np.inf]
        if top_k[i]:
            order = order[:top_k[i]]
        e = np.exp((row[order].astype(np.float64) - np.float64(row[order[0]])) / temperature[i])
        kept = len(e)
        if top_p[i] < 1.0:
            kept = int(np.searchsorted(np.cumsum(e), top_p[i] * e.sum())) + 1
        kept = min(kept, int((e >= min_p[i]).sum()))
        upto = np.cumsum(e[:kept])
        at = min(int(np.searchsorted(upto, u[i] * upto[-1], side="right")), kept - 1)
        tokens.append(int(order[at]))
        chances.append(float(e[at] / upto[-1]))
    return [torch.tensor(tokens, device=DEV), torch.tensor(chances, dtype=torch.float64, device=DEV)]


def work(case):
    if case["kind"] == "place":
        n, (_, new) = case["seqs"], _held(case)
        _, asked, returned, _ = _pages_of(case)
        return {"bytes": 12 * (sum(new) + case["padding"]) + 20 * n + 8 * (asked + returned), "flops": 8 * sum(new)}
    if case["kind"] == "embed":
        n = case["tokens"] * case["cols"]
        return {"bytes": n * ((1 if case["weight"] == "u8" else 2) + (4 if case["out"] == "f32" else 2)) + 12 * case["tokens"], "flops": 2 * n}
    if case["kind"] == "adapt":
        r, k, c, rank = case["rows"], case["k"], case["cols"], case["rank"]
        used, out = min(case["adapters"], case["seqs"]), 4 if case["out"] == "f32" else 2
        moved = r * k * (1 if case["x"] == "i8" else 2) + 2 * used * rank * (k + c) + r * c * ((4 if case["base"] == "f32" else 2) + out * (1 + case["mul"] + case["residual"]))
        return {"bytes": moved, "flops": 2 * r * rank * (k + c)}
    n = case["rows"] * case["vocabulary"]
    return {"bytes": n * (4 if case["dtype"] == "f32" else 2) + 16 * case["rows"], "flops": 8 * n}


if __name__ == "__main__":
    for c in listed() + [draw(random.Random(i)) for i in range(6)]:
        print(c, work(c))
