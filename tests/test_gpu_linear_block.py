"""The block of linear_block: all operators together, against the same formulas in 64 bits from the weights' own values."""
import math

import numpy as np
import pytest
import torch

from paper_2406_06237_amd import binding as B
from paper_2406_06237_amd import linear_block as L

pytestmark = pytest.mark.gpu

D_MODEL, D_FF, KV_HEADS = 512, 1376, 2


def plain(workload, xs):
    """The block in 64 bits for one sequence, nothing quantised but the weights."""
    w = {l.name: torch.from_numpy((s.astype(np.float64).reshape(l.shape) - l.zero_point) * l.channel_scales.astype(np.float64)[:, None])
         for l, s in zip(workload.layers, workload.symbols())}
    norm = lambda t: t / torch.sqrt((t * t).mean(-1, keepdim=True) + 1e-6)
    x = xs.cpu().double()
    n = norm(x)
    q, k, v = ((n @ w[m].T).view(len(x), -1, L.HEAD_DIM) for m in ("wq", "wk", "wv"))
    group = q.shape[1] // k.shape[1]
    scores = torch.einsum("thd,shd->hts", q, k.repeat_interleave(group, 1)) / math.sqrt(L.HEAD_DIM)
    scores = scores.masked_fill(torch.ones(len(x), len(x), dtype=torch.bool).triu(1), -math.inf)
    mixed = torch.einsum("hts,shd->thd", torch.softmax(scores, -1), v.repeat_interleave(group, 1)).reshape(len(x), -1)
    x = x + mixed @ w["wo"].T
    n = norm(x)
    gate = n @ w["wg"].T
    return x + (gate * torch.sigmoid(gate) * (n @ w["wu"].T)) @ w["wd"].T


# Rows of 8 bits are off by half a step of largest / 127 at most, that is by peak / 254 of their root mean square; peaks of normal rows of up to 1376 are
# about 4 times that, of products of two 10 times: 2 % for each of three kinds of rows and the cache's vectors (256 steps between the extremes), 5 % for the last.
# They add up, if nothing averages out, to 13 % of the block's two additions to x, which are not larger than the result.  4 bits in the cache are off
# by 1 / 30 of the range of about 6 times the root mean square: 20 % more of the first.
@pytest.mark.parametrize("bits,off", [(8, 0.13), (4, 0.33)])
def test_block(bits, off):
    workload = L.block_workload(D_MODEL, D_FF, KV_HEADS, seed=3)
    prompts, steps = [70, 1, 129], 2
    sequences = L.Sequences(len(prompts), max(prompts) + steps, seed=5)
    block = L.Block(workload, sequences.n_pages, bits)
    block.decode()
    want_symbols = np.concatenate(workload.symbols())
    np.testing.assert_array_equal(block.symbols[:len(want_symbols)].cpu().numpy(), want_symbols)
    g = torch.Generator().manual_seed(11)
    xs = [torch.randn(p + steps, D_MODEL, generator=g).to(torch.bfloat16) for p in prompts]
    got = [[] for _ in prompts]
    done = [0] * len(prompts)
    for new in [prompts] + [[1] * len(prompts)] * steps:                    # prompts together, then a token of each at a time
        x = torch.cat([xs[s][done[s]:done[s] + n] for s, n in enumerate(new)]).to("cuda:0")
        y = block.run(x, *sequences.append(new)).cpu()
        at = 0
        for s, n in enumerate(new):
            got[s].append(y[at:at + n])
            at += n
            done[s] += n
    assert block.container.read_status()[0] == 0 and int(block.cache.status[0]) == 0
    for s in range(len(prompts)):
        y, want = torch.cat(got[s]).double(), plain(workload, xs[s])
        rows = (y - want).norm(dim=-1) / want.norm(dim=-1)
        assert rows.max().item() < off, (s, rows.max().item())


def test_prompt_at_once_or_in_parts():
    """Rows of a product are alike whatever stands beside them, so that only attention's order of sums tells a prompt at once from one in parts."""
    workload = L.block_workload(D_MODEL, D_FF, KV_HEADS, seed=4)
    x = torch.randn(150, D_MODEL, generator=torch.Generator().manual_seed(12)).to(torch.bfloat16).to("cuda:0")
    results = []
    for parts in ([150], [100, 50], [149, 1]):
        sequences = L.Sequences(1, 150, seed=len(results))
        block = L.Block(workload, sequences.n_pages)
        block.decode()
        at, ys = 0, []
        for n in parts:
            ys.append(block.run(x[at:at + n].clone(), *sequences.append([n])))
            at += n
        results.append(torch.cat(ys).float())
    for other in results[1:]:
        # attention's weights have 11 bits and its output 8: a last bit of that and a symbol of the rows after it, of 8 bits each, twice over
        assert ((other - results[0]).norm(dim=-1) / results[0].norm(dim=-1)).max().item() < 4 * 2.0 ** -6


def test_status_of_a_page_that_is_not_there():
    workload = L.block_workload(D_MODEL, D_FF, KV_HEADS, seed=4)
    sequences = L.Sequences(1, 64)
    block = L.Block(workload, sequences.n_pages)
    block.decode()
    slots, pages, lengths, starts = sequences.append([3])
    x = torch.zeros(3, D_MODEL, dtype=torch.bfloat16, device="cuda:0")
    block.run(x, slots, pages + 7, lengths, starts)
    assert int(block.cache.status[0]) != 0
