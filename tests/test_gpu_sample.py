"""GPU: tokens drawn from logits by given random numbers: the same ones as a sorted list's in 64 bits."""
import numpy as np
import pytest
import torch

import serving_plain as P
from paper_2406_06237_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _tensor(v, dtype):
    return torch.tensor(v, dtype=dtype, device=DEV)


def _check(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """logits a tensor, u numbers, settings numbers or lists."""
    rows = logits.shape[0]
    each = lambda v: [float(torch.tensor(x, dtype=torch.float32)) if isinstance(x, float) else x for x in (v if isinstance(v, list) else [v] * rows)]  # noqa: E731
    given = lambda v, t: _tensor(v, t) if isinstance(v, list) else v  # noqa: E731
    f = torch.float32
    uniforms = _tensor(list(u), f)
    tokens, chances = B.sample(logits, uniforms, temperature=given(temperature, f), top_k=given(top_k, torch.int32), top_p=given(top_p, f), min_p=given(min_p, f))
    assert tokens.dtype == torch.int64 and chances.dtype == f
    for r, (row, x, t, k, p, m) in enumerate(zip(logits.float().cpu().numpy(), uniforms.tolist(), each(temperature), each(top_k), each(top_p), each(min_p))):
        token, chance = P.drawn(*P.kept(row, t, k, p, m), x)
        assert int(tokens[r]) == token, (r, int(tokens[r]), token, t, k, p, m, x)
        # one rounding to 32 bits, and weights whose polynomial leaves (ln2 / 128)^4 / 192 = 4.5e-12, in the token's and in the sum
        assert abs(float(chances[r]) - chance) <= chance * (2.0 ** -24 + 1e-11), (r, float(chances[r]), chance)
    return tokens


SETTINGS = [dict(), dict(temperature=0.6, top_p=0.9), dict(top_k=50), dict(top_k=7, top_p=0.8, min_p=0.05, temperature=1.3), dict(min_p=0.1), dict(top_p=0.3, temperature=2.0),
            dict(top_k=200, top_p=0.99)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocabulary,gap", [(1, 0), (2, 1), (7, 0), (64, 0), (1000, 3), (5003, 0), (8193, 1), (40001, 0), (131072, 0)])
def test_any_size(vocabulary, gap, dtype):
    g = torch.Generator(device=DEV).manual_seed(vocabulary)
    rows = 9
    logits = (torch.randn(rows, vocabulary + gap, device=DEV, generator=g) * 2.5).to(dtype)[:, gap:]
    logits += (torch.rand(rows, vocabulary, device=DEV, generator=g) < 20 / vocabulary).to(dtype) * 6
    u = torch.rand(rows, device=DEV, generator=g)
    u[0], u[1] = 0.0, 1 - 2.0 ** -24
    for s in SETTINGS:
        _check(logits, u.tolist(), **s)


def test_settings_of_each_row():
    g = torch.Generator(device=DEV).manual_seed(1)
    rows = 64
    logits = torch.randn(rows, 3001, device=DEV, generator=g) * 3
    rnd = lambda: torch.rand(rows, device=DEV, generator=g).tolist()  # noqa: E731
    _check(logits, rnd(), temperature=[0.0 if i % 7 == 0 else 0.2 + t for i, t in enumerate(rnd())], top_k=[int(k * 60) if i % 3 else -1 for i, k in enumerate(rnd())],
           top_p=[p if i % 4 else 1.0 for i, p in enumerate(rnd())], min_p=[m * 0.2 if i % 5 else 0.0 for i, m in enumerate(rnd())])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_all_alike(dtype):
    """More tokens of one logit than a list holds: the j-th of them by its number."""
    for n in (3, 511, 512, 513, 5000, 20000):
        logits = torch.full((8, n), 1.5, dtype=dtype, device=DEV)
        tokens = _check(logits, [(j + 0.5) / n for j in (0, 1, n // 3, n // 2, n - 2, n - 1, 0, n - 1)], top_k=[0, 0, 0, 0, 0, 0, 1, n])
        assert tokens.tolist() == [0, 1, n // 3, n // 2, n - 2, n - 1, 0, n - 1]
    logits = torch.full((3, 20000), -2.0, dtype=dtype, device=DEV)
    assert _check(logits, [0.99, 0.99, 0.99], top_k=[700, 5, 0], top_p=[1.0, 1.0, 0.25]).tolist() == [693, 4, 4950]


@pytest.mark.parametrize("spread", [1e-6, 1e-4, 3e-3, 0.05, 1.0])
def test_logits_close_together(spread):
    """Bins of more tokens than a list holds, of different logits and of equal ones."""
    g = torch.Generator(device=DEV).manual_seed(int(1 / spread))
    logits = torch.rand(12, 30000, device=DEV, generator=g) * spread + 0.25
    logits[4:8] = (logits[4:8] * 2 ** 12).round() / 2 ** 12
    logits[8:, ::3] = 0.25
    u = [0.0, 0.1, 0.37, 0.99] * 3
    for more in (dict(), dict(top_k=17000), dict(top_k=29999, top_p=0.7), dict(top_p=0.31), dict(min_p=0.99999), dict(top_k=600, top_p=0.5, min_p=0.2)):
        middles = []                                                   # u in the middle of what a token has
        for r in range(12):
            order, w = P.kept(logits[r].cpu().numpy(), 1.0, more.get("top_k", 0), float(np.float32(more.get("top_p", 1.0))), float(np.float32(more.get("min_p", 0.0))))
            j = int(u[r] * len(w))
            middles.append(float((np.cumsum(w)[j] - w[j] / 2) / w.sum()))
        _check(logits, middles, **more)


def test_masks():
    inf = float("inf")
    g = torch.Generator(device=DEV).manual_seed(4)
    logits = torch.randn(10, 700, device=DEV, generator=g)
    logits[:, 100:650] = -inf
    logits[1] = -inf
    logits[2] = -inf
    logits[2, 699] = -3e38                                             # one token is left, and the lowest number is no mask
    logits[3, 5] = float("nan")
    logits[4, [7, 20, 690]] = inf
    logits[5] = torch.finfo(torch.float32).min
    logits[6, :] = -inf
    logits[6, 3], logits[6, 600] = 3e38, -3e38                         # a difference beyond 32 bits
    logits[7] = 0.0
    logits[7, ::2] = -0.0
    u = [0.5, 0.5, 0.9, 0.5, 0.5, 0.7501, 0.99, 0.3333, 0.9, 0.1]
    for more in (dict(), dict(top_k=2), dict(top_p=0.4), dict(min_p=0.5), dict(temperature=0.0), dict(temperature=float("inf")), dict(temperature=1e-30), dict(temperature=1e30)):
        tokens = _check(logits, u, **more)
        assert int(tokens[1]) == int(tokens[3]) == -1 and int(tokens[2]) == 699
        if not more:
            assert int(tokens[4]) == 20 and int(tokens[5]) == int(0.7501 * 700) and int(tokens[7]) == int(0.3333 * 700)
    low = logits.to(torch.bfloat16)
    _check(low, u, top_k=40, top_p=0.9)


def test_borders():
    logits = torch.tensor([[0.0, 2.0, 1.0, 2.0, 1.0, -1.0]], device=DEV).expand(8, 6)
    last = 1 - 2.0 ** -24
    # the largest two are alike; of the next two the first is kept
    assert _check(logits, [0.0, last] * 4, top_k=[1, 1, 2, 2, 3, 3, 6, 100]).tolist() == [1, 1, 1, 3, 1, 2, 1, 5]
    assert _check(logits, [last] * 8, top_p=[0.0, 1e-9, 0.3, 0.5, 0.999, 1.0, 2.0, 1e9]).tolist() == [1, 1, 1, 3, 5, 5, 5, 5]
    assert _check(logits, [last] * 8, min_p=[1.0, 5.0, 0.9, 0.36, 0.1354, 0.0, 1e-30, 0.14]).tolist() == [3, 3, 3, 4, 4, 5, 5, 4]
    got, chances = B.sample(logits, _tensor([-1.0, 1.0, 2.0, float("nan"), float("inf"), -float("inf"), 0.5, 0.0], torch.float32))
    assert got.tolist()[:6] == [1, 5, 5, 1, 5, 1] and int(got[7]) == 1
    got, chances = B.sample(logits, _tensor([0.5] * 8, torch.float32), temperature=_tensor([-1.0, float("nan"), 0.0, 1, 1, 1, 1, 1], torch.float32),
                            top_p=_tensor([1, 1, 1, float("nan"), -1, 1, 1, 1], torch.float32), min_p=_tensor([0, 0, 0, 0, 0, float("nan"), -1, 0], torch.float32))
    assert got.tolist()[:3] == [-1, -1, 1] and chances.tolist()[:3] == [0, 0, 1] and got[3] == got[5] == got[6] == got[7] and int(got[4]) == 1


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocabulary", [1, 9, 4099, 8205, 33001])
def test_first_of_the_largest(vocabulary, dtype):
    """Without a temperature and with a top_k of 1, wherever the largest are: in the row's last elements, in two threads' or in two of a thread's."""
    g = torch.Generator(device=DEV).manual_seed(vocabulary)
    places = sorted({min(p, vocabulary - 1) for p in (0, 3, 4, 7, 8, 4095, 4096, 4100, 8191, 8192, vocabulary - 6, vocabulary - 2, vocabulary - 1) if p >= 0})
    logits = torch.randn(len(places), vocabulary, device=DEV, generator=g).to(dtype)
    for r, p in enumerate(places):
        logits[r, p:] = torch.where(torch.rand(vocabulary - p, device=DEV, generator=g) < 0.3, 9.0, logits[r, p:].float()).to(dtype)
        logits[r, p] = 9.0
    u = torch.rand(len(places), device=DEV, generator=g)
    for more in (dict(temperature=0.0), dict(top_k=1), dict(temperature=0.0, top_k=5, top_p=0.1, min_p=0.5)):
        tokens, chances = B.sample(logits, u, **more)
        assert tokens.tolist() == places and chances.tolist() == [1.0] * len(places)


def test_frequencies():
    """Uniforms that are spread evenly draw each token as often as its chance says, to one draw."""
    n = 4096
    row = torch.tensor([1.0, -0.5, 0.25, 2.0, 0.0], device=DEV)
    tokens, _ = B.sample(row.expand(n, 5), (torch.arange(n, device=DEV) + 0.5) / n, top_p=0.95)
    order, w = P.kept(row.tolist(), top_p=float(np.float32(0.95)))
    for token, weight in zip(order, w / w.sum()):
        assert abs(int((tokens == int(token)).sum()) - weight * n) <= 1


def test_large_vocabularies():
    """More than 2^18 tokens: fewer digits behind the point."""
    g = torch.Generator(device=DEV).manual_seed(2)
    logits = torch.randn(3, (1 << 18) + 5, device=DEV, generator=g) * 2
    _check(logits, [0.2, 0.5, 0.9], top_k=[0, 3000, 0], top_p=[1.0, 0.5, 0.7])


def test_into_an_output_on_another_stream():
    logits = torch.randn(5, 900, device=DEV)
    u = torch.rand(5, device=DEV)
    want, chances = B.sample(logits, u, top_k=20)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        into = torch.zeros(5, dtype=torch.int64, device=DEV)
        got, again = B.sample(logits, u, top_k=20, out=into)
    side.synchronize()
    assert got is into and torch.equal(into, want) and torch.equal(again, chances)
    assert B.sample(logits[:0], u[:0])[0].shape == (0,)


@pytest.mark.parametrize("rows,dtype", [(40, torch.float32), (700, torch.bfloat16)])
def test_top_p_by_the_bins_again_and_again(rows, dtype):
    """Rows whose top_p border and drawn token are found in the bins, by workgroups of each size: the same ones each time, and the formula's."""
    g = torch.Generator(device=DEV).manual_seed(rows)
    logits = (torch.randn(rows, 6001, device=DEV, generator=g) * 2.5).to(dtype)
    u = torch.rand(rows, device=DEV, generator=g)
    for more in (dict(top_p=0.9), dict(top_p=0.6, min_p=0.001), dict(top_p=0.97, top_k=900)):
        want = _check(logits[:40], u[:40].tolist(), **more)
        first = B.sample(logits, u, **more)
        assert torch.equal(first[0][:40], want)
        for _ in range(20):
            again = B.sample(logits, u, **more)
            assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocabulary", [3, 6, 60, 3000])
def test_uniforms_of_one_and_beyond_beside_both_borders(vocabulary, dtype):
    """The last token that is kept, where the weight's border lies in a bin that has no token, in one whose tokens weigh too little, and in one of which some are kept."""
    g = torch.Generator(device=DEV).manual_seed(vocabulary)
    uniforms = [1.0, 2.0, float("inf"), 1 - 2.0 ** -24, 0.0, 0.5]
    steps = torch.arange(vocabulary, device=DEV, dtype=torch.float32)
    logits = torch.stack([-steps, -6.0 * steps, -steps / 512, *(torch.randn(5, vocabulary, device=DEV, generator=g) * 2.5)]).to(dtype)
    logits = logits.repeat_interleave(len(uniforms), 0)
    # (no min_p is within the weights' error of a token's weight: logits of the first rows are whole numbers or 512ths)
    for top_p in (0.5, 0.99, 0.999):
        for min_p in (0.9995, 0.9, 0.3, 0.2, 0.05, 0.001):
            for more in (dict(), dict(top_k=vocabulary), dict(top_k=700)):
                _check(logits, uniforms * 8, top_p=top_p, min_p=min_p, **more)


def test_the_chance_of_a_light_token_is_the_same_by_the_list_and_by_the_bins():
    """The last of two tokens, down to 2^-40 of the first: its chance to one rounding, whether top_k lists them or not."""
    far = [1.0, 5.0, 10.0, 15.0, 19.4, 23.1, 27.7]
    logits = torch.tensor([[0.0, -f] for f in far], device=DEV)
    for more in (dict(), dict(top_k=2), dict(min_p=1e-13), dict(top_k=2, min_p=1e-13)):
        assert _check(logits, [1.0] * len(far), **more).tolist() == [1] * len(far)
