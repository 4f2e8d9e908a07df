"""GPU: low-rank adapters of many requests beside a product, against the formula in 64 bits."""
import pytest
import torch

import serving_plain as P
from operators_plain import HALF_ULP, assert_within
from paper_2406_06237_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


def _operands(rows, k, cols, rank, adapters, x="bf16", base=BF16, seed=0, gap=0):
    """With a gap, rows begin at any element."""
    g = torch.Generator(device=DEV).manual_seed(seed + rows * 7 + k)
    rnd = lambda *s: torch.randn(*s[:-1], s[-1] + gap, device=DEV, generator=g)[..., gap:]  # noqa: E731
    o = dict(base=rnd(rows, cols).to(base), a=(rnd(adapters, rank, k) / k ** 0.5).to(BF16), b=(rnd(adapters, cols, rank) / rank ** 0.5).to(BF16),
             ids=torch.randint(-1, adapters, (rows,), dtype=torch.int32, device=DEV, generator=g), scales=torch.rand(adapters, device=DEV, generator=g) + 0.5)
    if x == "i8":
        o.update(x=(rnd(rows, k) * 32).round().clamp(-127, 127).to(torch.int8), x_scales=(torch.rand(rows, device=DEV, generator=g) + 0.5) / 32)
    else:
        o["x"] = rnd(rows, k).to(BF16)
    return o


def _check(o, out="bf16", **epilogue):
    short = out == "bf16"
    want, error = P.adapt(**o, **epilogue, short=short)
    status = torch.zeros(2, dtype=torch.int32, device=DEV)
    got = B.adapt(**o, **epilogue, out_dtype=out, status=status)
    assert got.dtype == (BF16 if short else torch.float32)
    assert_within(got, want, error * 1.01 + want.abs() * HALF_ULP[got.dtype] * 1.01)
    assert status.tolist() == [0, 0]
    return got


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("x", ["bf16", "i8"])
@pytest.mark.parametrize("rows,k,cols,rank,adapters,gap", [
    (1, 64, 64, 16, 1, 0), (1, 1, 1, 1, 1, 0), (3, 63, 17, 5, 2, 1), (16, 512, 256, 8, 16, 0), (17, 200, 300, 13, 4, 3), (33, 1000, 65, 17, 3, 1), (64, 768, 520, 32, 48, 0),
    (40, 130, 1030, 33, 6, 0), (130, 320, 96, 64, 5, 0), (50, 4100, 70, 100, 2, 1), (20, 256, 257, 128, 3, 0), (18, 96, 40, 127, 2, 0), (200, 256, 130, 16, 3, 0), (256, 320, 200, 64, 40, 1), (1100, 192, 144, 24, 7, 0),
    (1031, 130, 259, 70, 3, 1), (1024, 64, 64, 120, 2, 0)])
def test_any_size(rows, k, cols, rank, adapters, gap, x, out):
    _check(_operands(rows, k, cols, rank, adapters, x, gap=gap, base=BF16 if rows % 2 else torch.float32), out)


@pytest.mark.parametrize("rows", [5, 1040])
@pytest.mark.parametrize("activation", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_epilogues(out, activation, rows):
    o = _operands(rows, 128, 75, 16, 4, "i8", torch.float32, seed=3)
    dt = BF16 if out == "bf16" else torch.float32
    mul, residual = (torch.randn(rows, 75, device=DEV).to(dt) for _ in range(2))
    plain = _check(o, out, activation=activation)
    _check(o, out, activation=activation, mul=mul)
    got = _check(o, out, activation=activation, mul=mul, residual=residual)
    into = mul.clone()
    assert torch.equal(B.adapt(**o, activation=activation, mul=into, residual=residual, out=into), got)
    base = o["base"].to(dt)
    want = B.adapt(**{**o, "base": base}, activation=activation, out_dtype=out)
    assert torch.equal(B.adapt(**{**o, "base": base}, activation=activation, out=base), want)
    assert plain.shape == want.shape


@pytest.mark.parametrize("rows", [2, 16, 40, 1100])
@pytest.mark.parametrize("ids", ["none", "one", "each", "runs", "beyond"])
def test_which_rows_have_which(rows, ids):
    o = _operands(rows, 100, 48, 12, 20, seed=rows)
    r = torch.arange(rows, device=DEV, dtype=torch.int32)
    o["ids"] = {"none": torch.full_like(r, -1), "one": torch.full_like(r, 3), "each": r % 20, "runs": r // 300 % 20, "beyond": torch.where(r % 3 == 0, 20 + r, r % 20)}[ids]
    want, error = P.adapt(**o)
    status = torch.zeros(2, dtype=torch.int32, device=DEV)
    got = B.adapt(**o, status=status)
    assert_within(got, want, error * 1.01 + want.abs() * 2.0 ** -8 * 1.01)
    beyond = int((o["ids"] >= 20).sum())
    assert status.tolist() == ([1, beyond] if beyond else [0, 0])
    if ids == "none":
        assert torch.equal(got, o["base"])
        empty = {**o, "a": o["a"][:0], "b": o["b"][:0], "scales": o["scales"][:0]}
        assert torch.equal(B.adapt(**empty), o["base"])


@pytest.mark.parametrize("rows", [24, 1030])
def test_other_rows_adapters_reach_nothing(rows):
    """Infinities and NaN in one request's adapter, or in its row of x, stay in its rows."""
    o = _operands(rows, 80, 40, 16, 4, seed=9)
    o["ids"] = torch.arange(rows, dtype=torch.int32, device=DEV) % 5 - 1
    want = B.adapt(**o)
    bad = {n: o[n].clone() for n in ("a", "b", "x", "scales")}
    bad["a"][1, 3, 5], bad["b"][1, :, 2], bad["b"][2] = float("inf"), float("nan"), float("-inf")
    bad["x"][9] = float("nan")
    got = B.adapt(**{**o, **bad})
    clean = (o["ids"] != 1) & (o["ids"] != 2) & (torch.arange(rows, device=DEV) != 9)
    assert torch.equal(got[clean], want[clean])
    assert not torch.isfinite(got[o["ids"] == 2]).any() and not torch.isfinite(got[o["ids"] == 1]).any()


def test_extremes_of_h():
    """h at the ends of the exponents' range: nothing becomes infinite that is a number."""
    o = dict(base=torch.zeros(4, 32, device=DEV), x=torch.ones(4, 32, dtype=BF16, device=DEV), a=torch.zeros(4, 3, 32, dtype=BF16, device=DEV),
             b=torch.zeros(4, 32, 3, dtype=BF16, device=DEV), ids=torch.arange(4, dtype=torch.int32, device=DEV), scales=torch.tensor([3.4e38, 1e-30, 1.0, 255.9], device=DEV))
    o["a"][:, :, 0], o["b"][:, :, 1] = 1.0, 0.5
    _check(o, "f32")
    _check(o, "bf16")


def test_a_long_row_of_adapters():
    """Adapters beyond 2^32 elements."""
    n, rank, k = 66, 128, 520000
    a = torch.zeros(n, rank, k, dtype=BF16, device=DEV)
    a[-1, 127, -1], a[0, 0, 0] = 2.0, 3.0
    b = torch.ones(n, 16, rank, dtype=BF16, device=DEV)
    x = torch.ones(2, k, dtype=BF16, device=DEV)
    got = B.adapt(torch.zeros(2, 16, device=DEV), x, a, b, torch.tensor([n - 1, 0], dtype=torch.int32, device=DEV), out_dtype="f32")
    assert (got[0] == 2).all() and (got[1] == 3).all()


@pytest.mark.parametrize("rows", [40, 1030])
def test_the_same_again(rows):
    o = _operands(rows, 700, 300, 16, 9, "i8")
    want = B.adapt(**o)
    for _ in range(5):
        assert torch.equal(B.adapt(**o), want)


@pytest.mark.parametrize("adapters", [1, 3, 4])
@pytest.mark.parametrize("rows", [63, 64, 65, 256, 257, 511, 512, 4097])
def test_where_another_kernel_begins(rows, adapters):
    for k in (100, 4200) if rows < 4000 else (100,):
        _check(_operands(rows, k, 136, 20, adapters, "i8"), "f32" if rows % 2 else "bf16")


@pytest.mark.parametrize("rows", [60, 200, 700])
def test_operands_of_one_row_for_all(rows):
    """Rows that lie on each other are read, each row's own as any."""
    o = _operands(rows, 256, 200, 16, 5, base=torch.float32)
    one = lambda dt, n: torch.randn(1, n, device=DEV).to(dt).expand(rows, n)  # noqa: E731
    o.update(base=one(torch.float32, 200), x=one(BF16, 256))
    _check(o, "bf16", mul=one(BF16, 200), residual=one(BF16, 200), activation="silu")


@pytest.mark.parametrize("rows", [60, 200, 700])
@pytest.mark.parametrize("cols", [75, 4100])
def test_into_each_operand_it_may(rows, cols):
    o = _operands(rows, 128, cols, 40, 11, "i8")
    mul, residual = (torch.randn(rows, cols, device=DEV).to(BF16) for _ in range(2))
    want = B.adapt(**o, mul=mul, residual=residual, activation="gelu")
    for which in ("base", "mul", "residual"):
        into = dict(o, mul=mul, residual=residual)
        into[which] = into[which].clone()
        assert torch.equal(B.adapt(**into, activation="gelu", out=into[which]), want)


@pytest.mark.parametrize("rank", [5, 8, 16, 40, 128])
@pytest.mark.parametrize("rows", [1, 60, 700])
def test_a_base_that_cancels_the_adapters(rows, rank):
    """h in whole numbers of 20 and 21 bits, one of them a column, and a base that leaves quarters: every step is exact in 32 bits, and so is the bf16 output."""
    k, cols, n = 60, 136, 3
    g = torch.Generator(device=DEV).manual_seed(rows + rank)
    whole = lambda lo, hi, *s: torch.randint(lo, hi, s, device=DEV, generator=g)  # noqa: E731
    x, a = whole(64, 128, rows, k), whole(128, 256, n, rank, k)
    of_column = torch.arange(cols, device=DEV) % rank
    b = torch.zeros(n, cols, rank, dtype=BF16, device=DEV)
    b[:, torch.arange(cols, device=DEV), of_column] = 1.0
    ids = torch.arange(rows, dtype=torch.int32, device=DEV) % (n + 1) - (0 if rows == 1 else 1)
    h = torch.stack([(x[r].cpu() * a[max(int(i), 0)].cpu()).sum(-1) for r, i in enumerate(ids.tolist())])[:, of_column.cpu()].to(DEV)
    left = whole(-64, 64, rows, cols) / 4
    base = left - h.float()
    assert h.max() < 2 ** 21 and torch.equal(base.double(), left.double() - h.double())
    o = dict(base=base, a=a.to(BF16), b=b, ids=ids)
    for of_x in (x.to(torch.int8), x.to(BF16)):
        got = B.adapt(**o, x=of_x)
        assert torch.equal(got, torch.where(ids[:, None] >= 0, left, base).to(BF16))
