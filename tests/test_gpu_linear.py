"""GPU: the product with its epilogue against the formula in 64 bits: both operand types, sizes on both sides of every tile, rows that begin
at any element, each activation, each operand of the epilogue."""
import pytest
import torch

import operators_plain as P
from paper_2406_06237_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _inputs(rows, cols, k, eight, seed=0, zero_point=8, most=15, pad=0, dtype=torch.bfloat16):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, device=DEV, generator=g)  # noqa: E731
    a = {}
    if eight:
        a["x"] = torch.randint(-128, 128, (rows, k + pad), device=DEV, generator=g).to(torch.int8)[:, pad:]
        a["weight"] = torch.randint(0, most + 1, (cols, k + pad), device=DEV, generator=g).to(torch.uint8)[:, pad:]
        a["x_scales"] = torch.rand(rows, device=DEV, generator=g) / 64
        a["channel_scales"] = torch.rand(cols, device=DEV, generator=g) / (most * k ** 0.5)
        a["zero_point"] = zero_point
    else:
        a["x"] = rnd(rows, k + pad).to(torch.bfloat16)[:, pad:]
        a["weight"] = (rnd(cols, k + pad) / k ** 0.5).to(torch.bfloat16)[:, pad:]
    a["bias"], a["mul"], a["residual"] = rnd(cols), rnd(rows, cols).to(dtype), rnd(rows, cols).to(dtype)
    return a


def _check(a, out_dtype, activation="none", what="", **more):
    want, error = P.linear(a["x"], a["weight"], a.get("x_scales"), a.get("zero_point", 0), more.get("scale", 1.0), a.get("channel_scales"), a.get("bias"),
                           activation, a.get("mul"), a.get("residual"))
    got = B.linear(**a, activation=activation, out_dtype=out_dtype, **more)
    P.assert_within(got, want, error + want.abs() * P.HALF_ULP[got.dtype], what)
    return got


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("k", [1, 15, 16, 64, 127, 128, 200, 1000, 4096])
def test_reductions(k, eight):
    for rows, cols, pad in ((1, 64, 0), (17, 65, 0), (70, 100, 3)):
        a = _inputs(rows, cols, k, eight, k, pad=pad)
        a["mul"] = a["residual"] = None
        _check(a, "f32", what=(rows, cols))


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("rows", [1, 2, 3, 8, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 100, 128, 129, 255, 256, 257, 300])
def test_rows(rows, eight):
    for cols, k in ((1, 64), (3, 300), (16, 128), (61, 96), (64, 256), (130, 520), (256, 2048), (515, 192)):
        _check(_inputs(rows, cols, k, eight, rows + cols), "bf16", what=(cols, k))


@pytest.mark.parametrize("activation", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("out_dtype", ["bf16", "f32"])
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("rows", [1, 24, 200])
def test_epilogues(rows, eight, out_dtype, activation):
    dtype = torch.float32 if out_dtype == "f32" else torch.bfloat16
    for n in range(8):
        a = _inputs(rows, 272, 256, eight, n, dtype=dtype)
        for i, name in enumerate(("bias", "mul", "residual")):
            if not n >> i & 1:
                a[name] = None
        _check(a, out_dtype, activation, what=n, scale=0.75)


@pytest.mark.parametrize("zero_point,most", [(0, 255), (255, 255), (128, 255), (100, 255), (8, 15), (1, 1), (64, 127)])
def test_zero_points(zero_point, most):
    for rows in (1, 20, 130, 300):
        for cols, k in ((80, 1000), (256, 1024)):
            a = _inputs(rows, cols, k, True, zero_point, zero_point, most)
            a["bias"] = a["mul"] = a["residual"] = a["x_scales"] = a["channel_scales"] = None
            want = P.wide(a["x"]) @ (P.wide(a["weight"]) - zero_point).T
            got = B.linear(**a, out_dtype="f32")
            assert torch.equal(got.cpu(), want.to(torch.float32))          # whole sums, rounded once


def test_sums_of_bytes_at_their_largest():
    k = 65536
    for q, z in ((0, 255), (255, 0), (255, 128)):
        x = torch.full((2, k), -128, dtype=torch.int8, device=DEV)
        w = torch.full((17, k), q, dtype=torch.uint8, device=DEV)
        got = B.linear(x, w, zero_point=z, out_dtype="f32")
        assert (got == float(-128 * (q - z) * k)).all()


@pytest.mark.parametrize("eight", [False, True])
def test_views_and_outputs_in_place(eight):
    for rows, cols, k in ((5, 192, 256), (140, 320, 384), (300, 512, 256)):
        a = _inputs(rows, cols, k, eight)
        want = B.linear(**a)
        wide = torch.zeros(rows, 2 * cols, dtype=torch.bfloat16, device=DEV)
        for name in ("mul", "residual"):
            wide[:, cols:] = a[name]
            assert torch.equal(B.linear(**{**a, name: wide[:, cols:]}), want)
            assert torch.equal(B.linear(**{**a, name: wide[:, cols:]}, out=wide[:, cols:]), want)
            assert (wide[:, :cols] == 0).all()
        far = torch.zeros(rows, k + 64, dtype=a["x"].dtype, device=DEV)
        far[:, 16:16 + k] = a["x"]
        assert torch.equal(B.linear(**{**a, "x": far[:, 16:16 + k]}), want)
        one = a["x"][:1].expand(rows, k)                               # every row the same memory
        assert torch.equal(B.linear(**{**a, "x": one}), B.linear(**{**a, "x": one.contiguous()}))


@pytest.mark.parametrize("rows", [1, 40, 300])
def test_infinities_stay_in_their_rows_and_channels(rows):
    a = _inputs(rows, 260, 256, False)
    a["mul"] = a["residual"] = None
    want = B.linear(**a, out_dtype="f32")
    a["x"][rows - 1, 9] = float("inf")
    a["weight"][7, 3] = float("nan")
    got = B.linear(**a, out_dtype="f32")
    assert torch.isnan(got[:, 7]).all() and not torch.isfinite(got[rows - 1]).any()
    keep = torch.ones_like(want, dtype=torch.bool)
    keep[:, 7] = keep[rows - 1] = False
    assert torch.equal(got[keep], want[keep])


def test_rows_beyond_32_bit_offsets():
    """A weight matrix of more than 4 GiB: its last rows, and a product of few and of many rows with it."""
    k, cols = 16384, 280000                                            # 4.6 GB of symbols
    w = torch.full((cols, k), 7, dtype=torch.uint8, device=DEV)
    w[-1, ::2] = 9
    for rows in (1, 300):
        x = torch.ones(rows, k, dtype=torch.int8, device=DEV)
        out = B.linear(x, w, zero_point=8, out_dtype="f32")
        assert (out[:, -1] == 0).all() and (out[:, :-1] == -k).all()
        del out


def test_nothing_to_do():
    x, w = torch.zeros(0, 64, dtype=torch.bfloat16, device=DEV), torch.zeros(32, 64, dtype=torch.bfloat16, device=DEV)
    assert B.linear(x, w).shape == (0, 32)
    assert B.linear(torch.zeros(3, 64, dtype=torch.bfloat16, device=DEV), w[:0]).shape == (3, 0)


@pytest.mark.parametrize("k", [7, 24])
def test_channels_beyond_one_dimension_of_a_launch(k):
    """More channels than 2^32 threads of few rows' kernel have: every one is written.  All have the same weights."""
    x, w = torch.randn(2, 1, k, device=DEV).to(torch.bfloat16)
    cols = (1 << 27) + 70
    out = torch.full((1, cols), float("nan"), dtype=torch.bfloat16, device=DEV)
    B.linear(x, w.expand(cols, k), out=out)
    want, error = P.linear(x, w)
    P.assert_within(out[:, :1], want, error + want.abs() * P.HALF_ULP[torch.bfloat16])
    assert (out == out[0, 0]).all()


@pytest.mark.parametrize("rows", [1, 40, 600])
def test_columns_of_one_buffer(rows):
    """Operands and output between each other's rows; an output over its operands is refused."""
    k, cols = 64, 72
    buffer = torch.randn(rows, k + 2 * cols, device=DEV).to(torch.bfloat16)
    w = torch.randn(cols, k, device=DEV).to(torch.bfloat16)
    x, out, residual = buffer[:, :k], buffer[:, k:k + cols], buffer[:, k + cols:]
    want = B.linear(x.clone(), w, residual=residual.clone())
    B.linear(x, w, residual=residual, out=out)
    assert torch.equal(out, want)
    for over in (buffer[:, k - 1:k - 1 + cols], buffer[:, k + cols - 8:k + 2 * cols - 8]):
        with pytest.raises(B.AnszpError, match="out of range"):
            B.linear(x, w, residual=residual, out=over)
    square = buffer[:, :k].contiguous()
    with pytest.raises(B.AnszpError, match="out of range"):
        B.linear(square, w[:k], out=square)
    with pytest.raises(B.AnszpError, match="out of range"):
        B.rms_norm(x, w[0], residual=residual[:, :k], total=buffer[:, 1:k + 1])
