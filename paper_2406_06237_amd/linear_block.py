"""One block of the linear stack at work: weights that arrive entropy-coded are decoded to their symbols and multiplied with as they are, 8 bits by
8 bits, between the norms, the quantised cache and the attention that a block of such matrices sits in.

    x' = x + wo . attention(wq . n, wk . n, wv . n)      n = norm(x)
    x'' = x' + wd . (silu(wg . m) * (wu . m))            m = norm(x')

One decode call, then thirteen calls a pass, whatever the number of tokens: a prompt's, one new token of each of many sequences, or both together
(attend takes a sequence's new tokens behind what its cache holds).  Rows are quantised by the call that makes them, or by quantise_rows
where that call has no such output.  The weights are seeded synthetic symbols (4 bits, Laplace at about 2.5 bit, a scale for each channel, as
workloads.config4 has them); there are no positions here, and without a vocabulary a step's input is the last output, normed.

With a vocabulary (--vocabulary) a step is a serving step: tokens are placed in the cache and looked up, rows go through the block, logits are one more
product, and the next tokens are drawn from them.  Nothing of it comes back to the host, so a step is captured into a graph once and replayed.  With
adapters (--adapters) each sequence has its own low-rank change to every matrix, added to the products by adapt.

With 4096 / 11008 and 8 heads in the cache (177 M weights in 56 MB) a decode takes 0.13 ms, prompts of 8 sequences with 6252 tokens 1.8 ms, a step of the 8
sequences 0.2 ms, most of which is the host's: its page lists and 13 calls from Python.  With a vocabulary of 32000 a captured step takes 0.19 ms, with eight adapters of
rank 16 0.29.

    python -m paper_2406_06237_amd.linear_block [--d-model N] [--d-ff N] [--prompt N] [--sequences N] [--steps N] [--bits 8|4] [--vocabulary N] [--adapters N]
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


def vocabulary_workload(d_model: int, vocabulary: int, seed: int = 0) -> W.Workload:
    """The vocabulary's matrices [vocabulary, d_model] as a workload: we, the rows of tokens, and wl, the weights of logits."""
    pmf = W.laplace_pmf(16, 8, W.laplace_beta_for_entropy(16, 8, 2.5))
    spread = math.sqrt(float((pmf * (np.arange(16) - 8.0) ** 2).sum()))
    layers = []
    for i, name in enumerate(("we", "wl")):
        own = W.BASE_SEED + 64 * seed + 57 + 2 * i
        u = (W.splitmix64(own, vocabulary) >> np.uint64(11)).astype(np.float64) / (1 << 53)
        scales = ((0.5 + u) / (math.sqrt(d_model) * spread)).astype(np.float32)
        layers.append(W.Layer(name, (vocabulary, d_model), 4, 8, float(scales[0]), pmf, own + 1, channel_len=d_model, channel_scales=scales))
    return W.Workload("vocabulary", layers, 12, 64, 65536, "bf16")


@dataclass
class Matrix:
    symbols: object          # uint8 [out, in]
    zero_point: int
    scales: object           # fp32 [out]

    def __call__(self, x, x_scales, adapters=None, ids=None, **epilogue):
        """The product with its epilogue; with adapters, and ids of each row's, what they add to it comes before the epilogue.  The product is in fp32 between the
        two calls, so that a row is rounded once, and one without an adapter has what it has where there are none."""
        if adapters is None:
            return B.linear(x, self.symbols, x_scales=x_scales, zero_point=self.zero_point, channel_scales=self.scales, **epilogue)
        base = B.linear(x, self.symbols, x_scales=x_scales, zero_point=self.zero_point, channel_scales=self.scales, out_dtype="f32")
        return B.adapt(base, x, adapters.a, adapters.b, ids, x_scales=x_scales, scales=adapters.scales, status=adapters.status, **epilogue)


@dataclass
class Adapter:
    """The adapters of one matrix: a bf16 [adapters, rank, in], b bf16 [adapters, out, rank], scales fp32 [adapters]."""
    a: object
    b: object
    scales: object
    status: object


def new_adapters(workload: W.Workload, count: int, rank: int, seed: int = 0, device="cuda:0") -> dict:
    """Random adapters for every matrix of the block, by its name, that change its outputs by about a quarter."""
    torch = B._torch()
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *shape: torch.randn(*shape, generator=g)
    status = torch.zeros(2, dtype=torch.int32, device=device)
    return {l.name: Adapter((rnd(count, rank, l.shape[1]) / math.sqrt(l.shape[1])).to(torch.bfloat16).to(device), (rnd(count, l.shape[0], rank) / math.sqrt(rank)).to(torch.bfloat16).to(device),
                            torch.full((count,), 0.25, device=device), status) for l in workload.layers}


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

    def run(self, x, slots, pages, lengths, starts, adapters=None, ids=None):
        """x bf16 [tokens, d_model], the new tokens of all sequences one sequence behind the other; slots, pages, lengths and starts as cache_write and
        attend take them.  adapters by the matrices' names, as new_adapters makes them, and ids int32 [tokens] which each token's is (-1: none).  Returns bf16 [tokens,
        d_model]."""
        tokens = x.shape[0]
        with_its = lambda name: dict(adapters=adapters[name], ids=ids) if adapters else {}
        n, s, _ = B.rms_norm(x, self.norms[0], out_dtype="i8")
        q, k, v = (getattr(self, name)(n, s, **with_its(name)) for name in ("wq", "wk", "wv"))
        B.cache_write(self.cache, k.view(tokens, -1, HEAD_DIM), v.view(tokens, -1, HEAD_DIM), slots)
        mixed = B.attend(q.view(tokens, -1, HEAD_DIM), self.cache, pages, lengths, starts).view(tokens, -1)
        n, s = B.quantise_rows(mixed)
        n, s, x = B.rms_norm(self.wo(n, s, **with_its("wo")), self.norms[1], residual=x, out_dtype="i8")
        gate = self.wg(n, s, activation="silu", **with_its("wg"))
        n, s = B.quantise_rows(self.wu(n, s, mul=gate, out=gate, **with_its("wu")))
        return self.wd(n, s, residual=x, out=x, **with_its("wd"))


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


class Serving:
    """Sequences that are served on the GPU from their tokens to their next ones: page tables, lengths and free pages live there, and a step asks nothing of the host."""

    def __init__(self, block: Block, words: W.Workload, count: int, most_tokens: int, adapters=None, seed: int = 0, device="cuda:0"):
        torch = B._torch()
        self.block, self.adapters, self.device, self.count = block, adapters, device, count
        container = B.to_device(B.pack_workload(words), device)
        symbols, at, matrices = B.alloc_out(container, "u8"), 0, []
        B.decode(container, symbols, "u8")
        for layer in words.layers:
            matrices.append(Matrix(symbols[at:at + layer.numel].view(layer.shape), layer.zero_point, torch.from_numpy(layer.channel_scales).to(device)))
            at += layer.numel
        self.words, self.logits = matrices
        width, n_pages = -(-most_tokens // PAGE_SIZE), block.cache.k.shape[0]
        self.pages = torch.zeros(count, width, dtype=torch.int32, device=device)
        self.lengths = torch.zeros(count, dtype=torch.int32, device=device)
        self.free = torch.from_numpy(np.random.default_rng(seed).permutation(n_pages).astype(np.int32)).to(device)
        self.n_free = torch.full((1,), n_pages, dtype=torch.int32, device=device)
        self.adapter_of = torch.full((count,), -1, dtype=torch.int32, device=device)

    def step(self, tokens, new, uniforms, ends=None, **settings):
        """tokens int64 [n], the new ones of all sequences one sequence behind the other, new int32 [sequences] how many each has; ends, as place_tokens takes it: sequences that begin
        anew.  settings: sample's.  Returns (the next token of each sequence int64, its chance, logits fp32 [sequences, vocabulary]).  A sequence without new tokens, and one that place_tokens
        refuses, as for lack of pages (its length stays, and the cache's status says so), has token -1 and a chance of 0; its logits mean nothing, and no
        token of it is to be given to a later step before those that it was refused."""
        torch = B._torch()
        if tokens.shape[0] == 0:
            raise ValueError("a step has one token at least")
        last = torch.empty_like(self.lengths)
        placed = B.place_tokens(self.pages, PAGE_SIZE, self.lengths, new, self.free, self.n_free, tokens.shape[0], ends=ends, lengths_out=self.lengths, n_free_out=self.n_free,
                                status=self.block.cache.status, last=last)
        x = B.embed(tokens, self.words.symbols, self.words.zero_point, self.words.scales, scale=math.sqrt(self.words.symbols.shape[1]), status=self.block.cache.status)
        ids = self.adapter_of[placed.owners.clamp_min(0)] if self.adapters else None
        y = self.block.run(x, placed.slots, self.pages, placed.lengths, placed.starts, self.adapters, ids)
        # (a sequence without a token, -1, has some row here)
        n, s, _ = B.rms_norm(y[last], self.block.norms[0], out_dtype="i8")
        logits = self.logits(n, s, out_dtype="f32")
        drawn, chances = B.sample(logits, uniforms, **settings)
        none = last < 0
        return drawn.masked_fill_(none, -1), chances.masked_fill_(none, 0.0), logits

    def captured_step(self, tokens, new, uniforms, ends=None, **settings):
        """The step as a graph that reads `tokens`, `new` and `uniforms`, and `ends` and settings that are tensors, each time it is replayed: (graph, its results).  The state is what it
        was before."""
        torch = B._torch()
        held = [self.pages, self.lengths, self.free, self.n_free, self.block.cache.status, *({id(a.status): a.status for a in self.adapters.values()}.values() if self.adapters else ())]
        state = [t.clone() for t in held]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            # (no sequence ends here: its pages would be dealt, and what the cache holds in them written over)
            self.step(tokens, new, uniforms, ends=None if ends is None else torch.zeros_like(ends), **settings)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            results = self.step(tokens, new, uniforms, ends=ends, **settings)
        for t, was in zip(held, state):
            t.copy_(was)
        return graph, results


def serve(a, workload: W.Workload, timed) -> int:
    """Prompts of random tokens, then a step captured once and replayed: main's work where there is a vocabulary."""
    torch = B._torch()
    most = a.prompt + a.steps + 1
    block = Block(workload, a.sequences * -(-most // PAGE_SIZE), a.bits)
    block.decode()
    words = vocabulary_workload(a.d_model, a.vocabulary)
    adapters = new_adapters(workload, a.adapters, 16) if a.adapters else None
    serving = Serving(block, words, a.sequences, most, adapters)
    if a.adapters:
        serving.adapter_of.copy_(torch.arange(a.sequences, dtype=torch.int32) % a.adapters)
    g = torch.Generator(device="cuda:0").manual_seed(1)
    counts = [max(1, a.prompt - s * a.prompt // (2 * a.sequences)) for s in range(a.sequences)]
    prompt = torch.randint(0, a.vocabulary, (sum(counts),), device="cuda:0", generator=g)
    uniforms = torch.rand(a.steps + 1, a.sequences, device="cuda:0", generator=g)
    new, settings = torch.tensor(counts, dtype=torch.int32, device="cuda:0"), dict(temperature=0.8, top_k=50, top_p=0.95)
    all_anew = torch.ones_like(new)
    serving.step(prompt, new, uniforms[0], **settings)       # (the first calls load the kernels; then the same sequences begin anew)
    tokens, _, _ = timed(f"prompts, {sum(counts)} tokens", lambda: serving.step(prompt, new, uniforms[0], ends=all_anew, **settings))
    one_each, u = torch.ones_like(new), uniforms[1].clone()
    graph, results = serving.captured_step(tokens, one_each, u, **settings)
    drawn = [tokens.clone()]

    def steps():
        for i in range(a.steps):
            u.copy_(uniforms[1 + i])
            graph.replay()
            tokens.copy_(results[0])
            drawn.append(tokens.clone())
    timed(f"{a.steps} captured steps of {a.sequences} tokens", steps)
    status = int(block.cache.status[0]) | (int(next(iter(adapters.values())).status[0]) if adapters else 0)
    print(f"status {status}, the first sequence's tokens {torch.stack(drawn)[:8, 0].tolist()} ...")
    return status


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--d-model", type=int, default=1024)
    ap.add_argument("--d-ff", type=int, default=2752)
    ap.add_argument("--kv-heads", type=int, default=2)
    ap.add_argument("--prompt", type=int, default=500, help="tokens of the longest prompt; the others are shorter")
    ap.add_argument("--sequences", type=int, default=8)
    ap.add_argument("--steps", type=int, default=32)
    ap.add_argument("--bits", type=int, default=8, choices=B.CACHE_BITS)
    ap.add_argument("--vocabulary", type=int, default=0, help="serve tokens of so large a vocabulary")
    ap.add_argument("--adapters", type=int, default=0, help="with a vocabulary: adapters of rank 16 that the sequences have in turn")
    a = ap.parse_args()
    torch = B._torch()

    workload = block_workload(a.d_model, a.d_ff, a.kv_heads)

    def timed(what, work):
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        result = work()
        torch.cuda.synchronize()
        print(f"{what:<52} {(time.perf_counter() - t0) * 1e3:9.3f} ms", flush=True)
        return result

    if a.vocabulary:
        return serve(a, workload, timed)
    sequences = Sequences(a.sequences, a.prompt + a.steps)
    block = Block(workload, sequences.n_pages, a.bits)

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
