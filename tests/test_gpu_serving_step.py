"""GPU: the serving step's operators together, as linear_block's Serving runs them: tokens placed, looked up, through the block with an adapter for each sequence, and drawn."""
import math

import numpy as np
import pytest
import torch

import serving_plain as P
from paper_2406_06237_amd import binding as B
from paper_2406_06237_amd import linear_block as L

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
D_MODEL, D_FF, KV_HEADS, VOCABULARY, SEQUENCES, RANK = 256, 704, 1, 1000, 3, 12
SETTINGS = dict(temperature=0.9, top_k=40, top_p=0.9, min_p=0.01)


def _serving(adapted, most=200, seed=3):
    workload = L.block_workload(D_MODEL, D_FF, KV_HEADS, seed=seed)
    block = L.Block(workload, SEQUENCES * -(-most // L.PAGE_SIZE))
    block.decode()
    adapters = L.new_adapters(workload, 2, RANK, seed=5) if adapted else None
    serving = L.Serving(block, L.vocabulary_workload(D_MODEL, VOCABULARY, seed=seed), SEQUENCES, most, adapters, seed=1)
    serving.adapter_of.copy_(torch.tensor([1, -1, 0], dtype=torch.int32))
    return workload, serving


def _ints(a):
    return torch.tensor(a, dtype=torch.int32, device=DEV)


def _plain_logits(workload, serving, tokens, adapter):
    """The last token's logits of one sequence in 64 bits, nothing quantised but the weights."""
    w = {l.name: torch.from_numpy((s.astype(np.float64).reshape(l.shape) - l.zero_point) * l.channel_scales.astype(np.float64)[:, None])
         for l, s in zip(workload.layers, workload.symbols())}
    if adapter >= 0 and serving.adapters:
        for name, its in serving.adapters.items():
            w[name] = w[name] + float(its.scales[adapter]) * its.b[adapter].cpu().double() @ its.a[adapter].cpu().double()
    we, wl = ((m.symbols.cpu().double() - m.zero_point) * m.scales.cpu().double()[:, None] for m in (serving.words, serving.logits))
    norm = lambda t: t / torch.sqrt((t * t).mean(-1, keepdim=True) + 1e-6)
    x = we[tokens] * math.sqrt(D_MODEL)
    n = norm(x)
    q, k, v = ((n @ w[m].T).view(len(x), -1, L.HEAD_DIM) for m in ("wq", "wk", "wv"))
    group = q.shape[1] // k.shape[1]
    scores = torch.einsum("thd,shd->hts", q, k.repeat_interleave(group, 1)) / math.sqrt(L.HEAD_DIM)
    scores = scores.masked_fill(torch.ones(len(x), len(x), dtype=torch.bool).triu(1), -math.inf)
    x = x + torch.einsum("hts,shd->thd", torch.softmax(scores, -1), v.repeat_interleave(group, 1)).reshape(len(x), -1) @ w["wo"].T
    n = norm(x)
    gate = n @ w["wg"].T
    x = x + (gate * torch.sigmoid(gate) * (n @ w["wu"].T)) @ w["wd"].T
    return norm(x[-1]) @ wl.T


# Rows of 8 bits are off by at most 13 % of the block's result, if nothing averages out (rows of normal numbers: half a step of largest / 127 is 2 % of their root mean square, three kinds
# of rows and the cache's vectors 2 % each, the last 5 %), and the last norm's row by 2 % more; the logits are a product of that.
@pytest.mark.parametrize("adapted", [False, True])
def test_a_prompt_and_steps(adapted):
    workload, serving = _serving(adapted)
    g = torch.Generator().manual_seed(8)
    history = [torch.randint(0, VOCABULARY, (n,), generator=g).tolist() for n in (70, 1, 129)]
    new = [len(t) for t in history]
    tokens = torch.tensor(sum(history, []), device=DEV)
    for step in range(3):
        u = torch.rand(SEQUENCES, generator=g).to(DEV)
        drawn, chances, logits = serving.step(tokens, _ints(new), u, **SETTINGS)
        assert serving.lengths.tolist() == [len(t) for t in history]
        for s, its in enumerate(history):
            want = _plain_logits(workload, serving, its, int(serving.adapter_of[s]))
            off = (logits[s].cpu().double() - want).norm() / want.norm()
            assert off < 0.15, (step, s, float(off))
            f = lambda v: float(np.float32(v))
            token, chance = P.drawn(*P.kept(logits[s].cpu().numpy(), f(0.9), 40, f(0.9), f(0.01)), float(u[s]))
            assert int(drawn[s]) == token and abs(float(chances[s]) - chance) <= chance * 2.0 ** -23
            its.append(token)
        new, tokens = [1] * SEQUENCES, drawn
    assert serving.block.cache.status.tolist() == [0, 0]
    if adapted:
        assert next(iter(serving.adapters.values())).status.tolist() == [0, 0]


@pytest.mark.parametrize("adapted", [False, True])
def test_captured_steps_are_the_eager_ones(adapted):
    """Replayed several times, with eager work between: the same tokens, chances and logits as without a graph."""
    results = []
    for captured in (False, True):
        _, serving = _serving(adapted)
        g = torch.Generator().manual_seed(9)
        tokens = torch.randint(0, VOCABULARY, (33 + 2 + 60,), generator=g).to(DEV)
        u = torch.rand(7, SEQUENCES, generator=g).to(DEV)
        tokens, _, _ = serving.step(tokens, _ints([33, 2, 60]), u[0], **SETTINGS)
        one, own, seen = _ints([1] * SEQUENCES), u[1].clone(), []
        if captured:
            graph, out = serving.captured_step(tokens, one, own, **SETTINGS)
        for i in range(1, 7):
            own.copy_(u[i])
            if captured:
                graph.replay()
            else:
                out = serving.step(tokens, one, own, **SETTINGS)
            seen += [t.clone() for t in out]
            tokens.copy_(out[0])
            torch.cuda.synchronize()
            torch.randn(1000, device=DEV).sum()                          # (the program's own work between replays)
        results.append([*seen, serving.lengths, serving.n_free, serving.pages])
    for eager, replayed in zip(*results):
        assert torch.equal(eager, replayed)


def test_sequences_end_and_begin_anew():
    """Places are refilled in a step: the others go on, pages come back, and the results are those of sequences that had the place for themselves."""
    _, serving = _serving(True)
    _, alone = _serving(True)
    g = torch.Generator().manual_seed(4)
    first, second = (torch.randint(0, VOCABULARY, (n,), generator=g).to(DEV) for n in (100 + 50 + 150, 1 + 80 + 1))
    u = torch.rand(2, SEQUENCES, generator=g).to(DEV)
    serving.step(first, _ints([100, 50, 150]), u[0], **SETTINGS)
    _, _, got = serving.step(second, _ints([1, 80, 1]), u[1], ends=_ints([0, 1, 0]), **SETTINGS)
    _, _, want = alone.step(second[1:81], _ints([0, 80, 0]), u[1], **SETTINGS)
    assert torch.equal(got[1], want[1]) and serving.lengths.tolist() == [101, 80, 151]
    held = [-(-n // L.PAGE_SIZE) for n in serving.lengths.tolist()]
    assert int(serving.n_free) == serving.block.cache.k.shape[0] - sum(held)
    pages = sum((serving.pages[s, :n].tolist() for s, n in enumerate(held)), []) + serving.free[:int(serving.n_free)].tolist()
    assert sorted(pages) == list(range(serving.block.cache.k.shape[0])) and serving.block.cache.status.tolist() == [0, 0]


def test_two_graphs_and_an_eager_call_do_not_share_memory():
    """Captured calls keep workspaces of their own: replayed in turn, with eager calls of other sizes between, each gives what it gave."""
    g = torch.Generator(device=DEV).manual_seed(6)
    rnd = lambda *s: torch.randn(*s, device=DEV, generator=g)  # noqa: E731
    graphs = []
    for rows in (5, 700):
        o = dict(base=rnd(rows, 300), x=rnd(rows, 500).to(torch.bfloat16), a=rnd(6, 20, 500).to(torch.bfloat16), b=rnd(6, 300, 20).to(torch.bfloat16),
                 ids=torch.randint(-1, 6, (rows,), dtype=torch.int32, device=DEV, generator=g))
        logits, u = rnd(rows, 3000) * 3, torch.rand(rows, device=DEV, generator=g)
        table, free = torch.zeros(rows, 3, dtype=torch.int32, device=DEV), torch.arange(3 * rows, dtype=torch.int32, device=DEV)
        held, n_free, new = torch.zeros(rows, dtype=torch.int32, device=DEV), _ints([3 * rows]), torch.full((rows,), 20, dtype=torch.int32, device=DEV)
        work = lambda o=o, l=logits, u=u, t=table, f=free, h=held, n=n_free, k=new, r=rows: [B.adapt(**o), *B.sample(l, u, top_p=0.8), *B.place_tokens(t, 16, h, k, f, n, 20 * r)]  # noqa: E731
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            work()
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = work()
        graphs.append((graph, out, [t.clone() for t in work()], work))
    for _ in range(3):
        for graph, out, want, work in graphs:
            for t in out:
                t.zero_()
            graph.replay()
            eager = work()
            torch.cuda.synchronize()
            for a, b, c in zip(out, want, eager):
                assert torch.equal(a, b) and torch.equal(c, b)


def test_both_of_the_bindings_paths_give_the_same(monkeypatch):
    def everything():
        g = torch.Generator(device=DEV).manual_seed(3)
        rnd = lambda *s: torch.randn(*s, device=DEV, generator=g)  # noqa: E731
        table, status = torch.full((2, 4), -1, dtype=torch.int32, device=DEV), _ints([0, 0])
        out = [*B.place_tokens(table, 16, _ints([0, 0]), _ints([20, 3]), _ints(list(range(9))), _ints([9]), 30, ends=_ints([0, 1]), status=status), table, status]
        tokens = torch.tensor([3, -1, 7, 20], device=DEV)
        symbols = torch.randint(0, 16, (9, 70), device=DEV, generator=g).to(torch.uint8)
        out += [B.embed(tokens, symbols, 7, rnd(9), 2.0, status=status), B.embed(tokens, rnd(9, 70).to(torch.bfloat16), out_dtype="f32"), status]
        into = torch.zeros(4, 100, dtype=torch.bfloat16, device=DEV)
        B.embed(tokens, symbols, out=into[:, 5:75])
        x = torch.randint(-100, 100, (4, 64), device=DEV, generator=g).to(torch.int8)
        o = dict(a=rnd(3, 10, 64).to(torch.bfloat16), b=rnd(3, 70, 10).to(torch.bfloat16), ids=_ints([2, -1, 0, 9]), x_scales=rnd(4), scales=rnd(3), status=status)
        out += [into, B.adapt(out[-3], x, **o, activation="gelu", residual=rnd(4, 70).to(torch.bfloat16)), B.adapt(rnd(4, 70), x, **o, mul=rnd(4, 70), out_dtype="f32"), status]
        logits = rnd(4, 500) * 3
        out += [*B.sample(logits, torch.rand(4, device=DEV, generator=g), 0.7, 20, 0.9, 0.01), *B.sample(logits.to(torch.bfloat16), torch.rand(4, device=DEV, generator=g), top_p=rnd(4).abs(),
                                                                                                         temperature=rnd(4).abs(), min_p=rnd(4).abs() / 9, top_k=_ints([0, 3, 400, 1]))]
        return [t.clone() for t in out]

    assert B._operator_calls()
    native = everything()
    monkeypatch.setattr(B, "_host", False)
    for a, b in zip(native, everything()):
        assert a.dtype == b.dtype and a.shape == b.shape and torch.equal(a, b)


@pytest.mark.parametrize("rows", [5, 90, 600])
def test_a_row_without_an_adapter_is_the_same_beside_adapters(rows):
    """To the bit, with each epilogue that the block has."""
    workload = L.block_workload(D_MODEL, D_FF, KV_HEADS)
    block = L.Block(workload, 1)
    block.decode()
    adapters = L.new_adapters(workload, 3, RANK)
    g = torch.Generator(device=DEV).manual_seed(rows)
    rnd = lambda *s: torch.randn(*s, device=DEV, generator=g)  # noqa: E731
    ids = torch.arange(rows, dtype=torch.int32, device=DEV) % 4 - 1
    without = ids < 0
    for name in ("wq", "wg", "wu", "wd"):
        matrix = getattr(block, name)
        out, k = matrix.symbols.shape
        n, s = B.quantise_rows(rnd(rows, k))
        beside = rnd(rows, out).to(torch.bfloat16)
        epilogue = {"wq": {}, "wg": dict(activation="silu"), "wu": dict(mul=beside), "wd": dict(residual=beside)}[name]
        want, got = matrix(n, s, **epilogue), matrix(n, s, adapters=adapters[name], ids=ids, **epilogue)
        assert torch.equal(got[without], want[without]) and not torch.equal(got, want)


def test_a_sequence_without_an_adapter_has_the_logits_it_has_alone():
    _, adapted = _serving(True)
    _, plain = _serving(False)
    g = torch.Generator().manual_seed(2)
    tokens, u = torch.randint(0, VOCABULARY, (20 + 90 + 3,), generator=g).to(DEV), torch.rand(SEQUENCES, generator=g).to(DEV)
    got, want = (serving.step(tokens, _ints([20, 90, 3]), u, **SETTINGS)[2] for serving in (adapted, plain))
    assert torch.equal(got[1], want[1]) and not torch.equal(got[0], want[0]) and not torch.equal(got[2], want[2])


def test_a_sequence_for_which_no_page_is_left():
    """It has no token, the others have theirs, and it goes on once there are pages."""
    _, serving = _serving(False, most=300)
    _, other = _serving(False, most=300)
    g = torch.Generator().manual_seed(12)
    tokens = torch.randint(0, VOCABULARY, (100 + 64 + 30,), generator=g).to(DEV)
    u = torch.rand(3, SEQUENCES, generator=g).to(DEV)
    for s in (serving, other):
        s.step(tokens, _ints([100, 64, 30]), u[0], **SETTINGS)
    kept = int(serving.n_free)
    serving.n_free.zero_()
    one = torch.tensor([7, 8, 9], device=DEV)
    got, chances, logits = serving.step(one, _ints([1, 1, 1]), u[1], **SETTINGS)
    want = other.step(one, _ints([1, 1, 1]), u[1], **SETTINGS)
    # (64 tokens fill a page, so the second sequence needs another one)
    assert got.tolist() == [int(want[0][0]), -1, int(want[0][2])] and chances.tolist() == [float(want[1][0]), 0.0, float(want[1][2])]
    assert serving.lengths.tolist() == [101, 64, 31] and serving.block.cache.status.tolist() == [1, 1] and torch.equal(logits[0], want[2][0]) and torch.equal(logits[2], want[2][2])
    serving.n_free.fill_(kept)
    got, chances, logits = serving.step(one[1:2], _ints([0, 1, 0]), u[1], **SETTINGS)
    assert got.tolist() == [-1, int(want[0][1]), -1] and chances.tolist() == [0.0, float(want[1][1]), 0.0] and serving.lengths.tolist() == [101, 65, 31]
    # more tokens than the row of the table has room for, and more than are given
    got, chances, _ = serving.step(tokens[:30], _ints([1000, 3, 5]), u[2], **SETTINGS)
    assert got.tolist() == [-1, -1, -1] and chances.tolist() == [0.0] * 3 and serving.lengths.tolist() == [101, 65, 31]


def test_a_captured_step_in_which_sequences_end():
    """`ends` is read at each replay, and what is captured leaves the sequences that it names as they were."""
    results = []
    for captured in (False, True):
        _, serving = _serving(True)
        g = torch.Generator().manual_seed(21)
        first, after = (torch.randint(0, VOCABULARY, (n,), generator=g).to(DEV) for n in (60 + 70 + 5, SEQUENCES))
        u = torch.rand(6, SEQUENCES, generator=g).to(DEV)
        serving.step(first, _ints([60, 70, 5]), u[0], **SETTINGS)
        tokens, new, own, ends, seen = after.clone(), _ints([1, 1, 1]), u[1].clone(), _ints([1, 1, 0]), []
        if captured:
            # (no page is left but those of the sequences that would end)
            kept = serving.n_free.clone()
            serving.n_free.zero_()
            graph, out = serving.captured_step(tokens, new, own, ends=ends, **SETTINGS)
            assert serving.block.cache.status.tolist() == [0, 0] and serving.n_free.tolist() == [0] and serving.lengths.tolist() == [60, 70, 5]
            serving.n_free.copy_(kept)
        for i, which in enumerate(([0, 0, 0], [0, 1, 0], [0, 0, 0], [1, 0, 1], [0, 0, 0])):
            own.copy_(u[1 + i])
            ends.copy_(_ints(which))
            if captured:
                graph.replay()
            else:
                out = serving.step(tokens, new, own, ends=ends, **SETTINGS)
            seen += [t.clone() for t in out]
            tokens.copy_(out[0])
            torch.cuda.synchronize()
        results.append([*seen, serving.lengths, serving.n_free, serving.pages, serving.free[:int(serving.n_free)], serving.block.cache.status])
    for eager, replayed in zip(*results):
        assert torch.equal(eager, replayed)
    assert results[0][-1].tolist() == [0, 0]


def test_a_step_of_no_tokens_is_refused_before_it_changes_anything():
    _, serving = _serving(False)
    g = torch.Generator().manual_seed(1)
    tokens, u = torch.randint(0, VOCABULARY, (9,), generator=g).to(DEV), torch.rand(SEQUENCES, generator=g).to(DEV)
    serving.step(tokens, _ints([3, 3, 3]), u)
    state = [t.clone() for t in (serving.pages, serving.lengths, serving.free, serving.n_free)]
    with pytest.raises(ValueError, match="one token at least"):
        serving.step(tokens[:0], _ints([0, 0, 0]), u, ends=_ints([1, 0, 0]))
    assert all(torch.equal(a, b) for a, b in zip(state, (serving.pages, serving.lengths, serving.free, serving.n_free)))


def test_operands_that_ask_for_a_gradient_get_none():
    """As the docstrings say: the results are apart from autograd, and the operands' own gradients stay empty."""
    g = torch.Generator(device=DEV).manual_seed(1)
    rnd = lambda *s: torch.randn(*s, device=DEV, generator=g)  # noqa: E731
    a, b, base = rnd(2, 8, 64).to(torch.bfloat16).requires_grad_(), rnd(2, 40, 8).to(torch.bfloat16).requires_grad_(), rnd(3, 40).requires_grad_()
    logits, words = rnd(3, 90).requires_grad_(), rnd(9, 40).to(torch.bfloat16).requires_grad_()
    results = [B.adapt(base, rnd(3, 64).to(torch.bfloat16), a, b, _ints([0, 1, -1])), B.embed(torch.tensor([1, 2], device=DEV), words), *B.sample(logits, torch.rand(3, device=DEV))]
    assert not any(t.requires_grad for t in results) and all(t.grad is None for t in (a, b, base, logits, words))
    assert all("No gradient" in function.__doc__ for function in (B.adapt, B.embed, B.sample))


@pytest.mark.parametrize("adapted", [False, True])
def test_a_step_is_what_its_calls_give_one_by_one(adapted):
    """To the bit: page tables and slots from the host, tokens looked up by the formula, ids row by row, the last rows by their numbers."""
    workload, serving = _serving(adapted)
    block, sequences = L.Block(workload, SEQUENCES * -(-200 // L.PAGE_SIZE)), L.Sequences(SEQUENCES, 200)
    block.decode()
    g = torch.Generator().manual_seed(31)
    which = serving.adapter_of.tolist()
    for new in ([70, 1, 129], [1, 1, 1], [3, 64, 20], [1, 0, 1]):
        tokens, u = torch.randint(0, VOCABULARY, (sum(new),), generator=g).to(DEV), torch.rand(SEQUENCES, generator=g).to(DEV)
        drawn, chances, got = serving.step(tokens, _ints(new), u, **SETTINGS)
        x = P.embed(tokens, serving.words.symbols, serving.words.zero_point, serving.words.scales, math.sqrt(D_MODEL)).to(torch.bfloat16).to(DEV)
        ids = _ints([which[s] for s, n in enumerate(new) for _ in range(n)])
        y = block.run(x, *sequences.append(new), serving.adapters, ids)
        there = [s for s, n in enumerate(new) if n]
        n, s, _ = B.rms_norm(y[[sum(new[:s + 1]) - 1 for s in there]], block.norms[0], out_dtype="i8")
        want = serving.logits(n, s, out_dtype="f32")
        assert torch.equal(got[there], want)
        tokens, its = B.sample(want, u[there], **SETTINGS)
        assert torch.equal(drawn[there], tokens) and torch.equal(chances[there], its)
