"""One block of the linear stack at work: weights that arrive entropy-coded are decoded to their symbols and multiplied with as they are, 8 bits by
8 bits, between the norms, the quantised cache and the attention that a block of such matrices sits in.

    x' = x + wo . attention(wq . n, wk . n, wv . n)      n = norm(x)
    x'' = x' + wd . (silu(wg . m) * (wu . m))            m = norm(x')

One decode call, then thirteen calls a pass, whatever the number of tokens: a prompt's, one new token of each of many sequences, or both together
(attend takes a sequence's new tokens behind what its cache holds).  Rows are quantised by the call that makes them, or by quantise_rows
where that call has no such output.  The weights are seeded synthetic symbols (4 bits, Laplace at about 2.5 bit, a scale for each channel, as
workloads.config4 has them); there are no positions and no vocabulary here: a step's input is the last output, normed.

With 4096 / 11008 and 8 heads in the cache (177 M weights in 56 MB) a decode takes 0.13 ms, prompts of 8 sequences with 6252 tokens 1.8 ms, a step of the 8
sequences 0.2 ms, most of which is the host's: its page lists and 13 calls from Python.

    python -m paper_2406_06237_amd.linear_block [--d-model N] [--d-ff N] [--prompt N] [--sequences N] [--steps N] [--bits 8|4]
"""
import argparse
import math
import time
from dataclasses import dataclass

import numpy as np

from . import binding as B
from . import workloads as W

HEAD_DIM, PAGE_SIZE = 128, 64


def block_workload(d_model: int, d_ff: int, kv_heads: int, seed: int = 0) -> W.Workload:
    """The block's matrices [out, in] as a workload: wq, wk, wv, wo, wg, wu, wd; scales keep outputs about as large as inputs."""
    pmf = W.laplace_pmf(16, 8, W.laplace_beta_for_entropy(16, 8, 2.5))
    spread = math.sqrt(float((pmf * (np.arange(16) - 8.0) ** 2).sum()))
    kv = kv_heads * HEAD_DIM
    layers = []
    for i, (name, rows, cols) in enumerate((("wq", d_model, d_model), ("wk", kv, d_model), ("wv", kv, d_model), ("wo", d_model, d_model),
                                            ("wg", d_ff, d_model), ("wu", d_ff, d_model), ("wd", d_model, d_ff))):
        own = W.BASE_SEED + 64 * seed + 8 * i
        u = (W.splitmix64(own, rows) >> np.uint64(11)).astype(np.float64) / (1 << 53)
        scales = ((0.5 + u) / (math.sqrt(cols) * spread)).astype(np.float32)
        layers.append(W.Layer(name, (rows, cols), 4, 8, float(scales[0]), pmf, own + 1, channel_len=cols, channel_scales=scales))
    return W.Workload("linear_block", layers, 12, 64, 65536, "bf16")


@dataclass
class Matrix:
    symbols: object          # uint8 [out, in]
    zero_point: int
    scales: object           # fp32 [out]

    def __call__(self, x, x_scales, **epilogue):
        return B.linear(x, self.symbols, x_scales=x_scales, zero_point=self.zero_point, channel_scales=self.scales, **epilogue)


class Block:
    """A block on `device` with its own cache.  Sequences share the cache's pages by a page table."""

    def __init__(self, workload: W.Workload, n_pages: int, bits: int = 8, device="cuda:0"):
        torch = B._torch()
        self.container = B.to_device(B.pack_workload(workload), device)
        self.symbols = B.alloc_out(self.container, "u8")
        at = 0
        for layer in workload.layers:
            own = self.symbols[at:at + layer.numel].view(layer.shape)
            setattr(self, layer.name, Matrix(own, layer.zero_point, torch.from_numpy(layer.channel_scales).to(device)))
            at += layer.numel
        d_model = self.wq.symbols.shape[1]
        self.norms = [torch.ones(d_model, dtype=torch.float32, device=device) for _ in range(2)]
        self.cache = B.new_kv_cache(n_pages, PAGE_SIZE, self.wk.symbols.shape[0] // HEAD_DIM, HEAD_DIM, bits, device)

    def decode(self):
        """The block's symbols from its compressed weights: after this `run` may be called any number of times."""
        B.decode(self.container, self.symbols, "u8")

    def run(self, x, slots, pages, lengths, starts):
        """x bf16 [tokens, d_model], the new tokens of all sequences one sequence behind the other; slots, pages, lengths and starts as cache_write and
        attend take them.  Returns bf16 [tokens, d_model]."""
        tokens = x.shape[0]
        n, s, _ = B.rms_norm(x, self.norms[0], out_dtype="i8")
        q, k, v = self.wq(n, s), self.wk(n, s), self.wv(n, s)
        B.cache_write(self.cache, k.view(tokens, -1, HEAD_DIM), v.view(tokens, -1, HEAD_DIM), slots)
        mixed = B.attend(q.view(tokens, -1, HEAD_DIM), self.cache, pages, lengths, starts).view(tokens, -1)
        n, s = B.quantise_rows(mixed)
        n, s, x = B.rms_norm(self.wo(n, s), self.norms[1], residual=x, out_dtype="i8")
        gate = self.wg(n, s, activation="silu")
        n, s = B.quantise_rows(self.wu(n, s, mul=gate, out=gate))
        return self.wd(n, s, residual=x, out=x)


class Sequences:
    """Sequences of different lengths over one cache: pages are dealt out in a shuffled order, as they are after some time of use."""

    def __init__(self, count: int, most_tokens: int, seed: int = 0, device="cuda:0"):
        torch = B._torch()
        width = -(-most_tokens // PAGE_SIZE)
        self.n_pages, self.device = count * width, device
        order = np.random.default_rng(seed).permutation(self.n_pages).astype(np.int32)
        self.pages = torch.from_numpy(order.reshape(count, width)).to(device)
        self.lengths = [0] * count

    def append(self, new):
        """new[s] tokens more for each sequence s: (slots, pages, lengths, starts) for Block.run."""
        torch = B._torch()
        table, slots = self.pages.cpu().numpy(), []
        for s, n in enumerate(new):
            at = np.arange(self.lengths[s], self.lengths[s] + n)
            slots.append(table[s, at // PAGE_SIZE].astype(np.int64) * PAGE_SIZE + at % PAGE_SIZE)
            self.lengths[s] += n
        ints = lambda a: torch.tensor(a, dtype=torch.int32, device=self.device)
        return torch.from_numpy(np.concatenate(slots)).to(self.device), self.pages, ints(self.lengths), ints([0, *np.cumsum(new)])


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--d-model", type=int, default=1024)
    ap.add_argument("--d-ff", type=int, default=2752)
    ap.add_argument("--kv-heads", type=int, default=2)
    ap.add_argument("--prompt", type=int, default=500, help="tokens of the longest prompt; the others are shorter")
    ap.add_argument("--sequences", type=int, default=8)
    ap.add_argument("--steps", type=int, default=32)
    ap.add_argument("--bits", type=int, default=8, choices=B.CACHE_BITS)
    a = ap.parse_args()
    torch = B._torch()

    workload = block_workload(a.d_model, a.d_ff, a.kv_heads)
    sequences = Sequences(a.sequences, a.prompt + a.steps)
    block = Block(workload, sequences.n_pages, a.bits)

    def timed(what, work):
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        result = work()
        torch.cuda.synchronize()
        print(f"{what:<52} {(time.perf_counter() - t0) * 1e3:9.3f} ms", flush=True)
        return result

    size = block.container.host.compressed_bytes()
    print(f"{workload.numel / 1e6:.1f} M weights in {size / 1e6:.2f} MB ({8 * size / workload.numel:.2f} bit each)")
    block.decode()
    timed("decode to symbols", block.decode)

    new = [max(1, a.prompt - s * a.prompt // (2 * a.sequences)) for s in range(a.sequences)]
    x = torch.randn(sum(new), a.d_model, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to("cuda:0")
    places = sequences.append(new)
    block.run(x.clone(), *places)                            # (the first calls load the kernels; the same tokens in the same slots again)
    y = timed(f"prompts, {sum(new)} tokens", lambda: block.run(x.clone(), *places))
    last = y[places[3][1:].long() - 1]

    def step():
        nonlocal last
        x, _, _ = B.rms_norm(last, block.norms[0])
        last = block.run(x, *sequences.append([1] * a.sequences))
    step()
    timed(f"{a.steps - 1} steps of {a.sequences} tokens", lambda: [step() for _ in range(a.steps - 1)])
    bits, _ = block.container.read_status()
    cache_bits = int(block.cache.status[0])
    print(f"status {bits | cache_bits}, output's root mean square {float(last.float().square().mean().sqrt()):.3f}")
    return bits | cache_bits


if __name__ == "__main__":
    raise SystemExit(main())
