"""GPU: the root-mean-square norm against the formula in 64 bits, at every width class of its kernels, from rows that begin at any
element, with and without a residual, in fp32, bf16 and 8 bits."""
import pytest
import torch

import operators_plain as P
from paper_2406_06237_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-5
# sums over 32 elements a thread, 6 exchanges in a wavefront and 15 more
SUM = 2.0 ** -24 * 64


def _inputs(rows, cols, dtype, seed=0, pad=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(rows, cols + pad, device=DEV, generator=g).to(dtype)[:, pad:]
    r = (3 * torch.randn(rows, cols + pad, device=DEV, generator=g)).to(dtype)[:, :cols]
    return x, r, (1 + 0.3 * torch.randn(cols, device=DEV, generator=g)).to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cols", [1, 7, 8, 64, 512, 513, 1000, 1024, 1025, 2048, 4096, 4099, 8192, 11008, 16384, 16391, 40000])
def test_widths(cols, dtype):
    for rows, pad, residual in ((1, 0, True), (3, 0, False), (5, 1, True), (66, 0, True)):
        x, r, w = _inputs(rows, cols, dtype, cols + rows, pad)
        r = r if residual else None
        y, h = P.rms_norm(x, w, EPS, r)
        for out_dtype in ("f32", "bf16", "i8"):
            out, scales, total = B.rms_norm(x, w, EPS, residual=r, out_dtype=out_dtype)
            if residual:
                assert torch.equal(total, (x.float() + r.float()).to(dtype))
            else:
                assert total is None
            if out_dtype == "i8":
                most = y.abs().amax(-1)
                P.assert_within(scales, most / 127, most / 127 * SUM)
                P.assert_within(out.double() * scales.double()[:, None], y, (most / 127 * (0.5 + 127 * 2 * SUM))[:, None].expand_as(y))
                assert out.abs().max().item() == 127 and (out >= -127).all()
            else:
                assert scales is None
                P.assert_within(out, y, y.abs() * (SUM + P.HALF_ULP[out.dtype]))


@pytest.mark.parametrize("cols", [64, 4096, 40000])
def test_the_sum_may_replace_its_inputs(cols):
    x, r, w = _inputs(9, cols, torch.bfloat16)
    want, _, total = B.rms_norm(x, w, EPS, residual=r)
    for which in (0, 1):
        a, b = x.clone(), r.clone()
        out, _, same = B.rms_norm(a, w, EPS, residual=b, total=(a, b)[which])
        assert same.data_ptr() == (a, b)[which].data_ptr()
        assert torch.equal(same, total) and torch.equal(out, want)


def test_rows_without_a_number_and_rows_of_zeros():
    for cols in (64, 4096, 40000):
        x, _, w = _inputs(6, cols, torch.float32)
        x[1] = 0
        x[2, 5] = float("nan")
        x[3, cols - 1] = float("inf")
        x[4] = 1e-30
        out, scales, _ = B.rms_norm(x, w, EPS, out_dtype="i8")
        q, by = B.quantise_rows(x)
        for symbols, s in ((out, scales), (q, by)):
            assert torch.isnan(s[[2, 3]]).all() and torch.isfinite(s[[0, 1, 4, 5]]).all()
            assert (symbols[1:4] == 0).all() and s[1] == 0 and s[4] > 0 and symbols[4].abs().max() == 127
        out, _, _ = B.rms_norm(x, w, EPS, out_dtype="f32")
        assert (out[1] == 0).all() and torch.isnan(out[2]).all()
        assert torch.isnan(out[3, cols - 1]) and (out[3, : cols - 1] == 0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cols", [1, 100, 4096, 11008, 20000])
def test_rows_in_eight_bits_without_a_norm(cols, dtype):
    x, _, _ = _inputs(7, cols, dtype, pad=3)
    q, scales = B.quantise_rows(x)
    most = P.wide(x).abs().amax(-1)
    P.assert_within(scales, most / 127, most / 127 * 2.0 ** -22)
    P.assert_within(q.double() * scales.double()[:, None], P.wide(x), (most / 127 * (0.5 + 2.0 ** -14))[:, None].expand_as(x.cpu()))


def test_weights_of_the_other_type_and_rows_many():
    x, r, w = _inputs(70001, 64, torch.bfloat16)
    want, _, _ = B.rms_norm(x, w, EPS, residual=r)
    got, _, _ = B.rms_norm(x, w.float(), EPS, residual=r)
    assert torch.equal(got, want)
    y, _ = P.rms_norm(x, w, EPS, r)
    P.assert_within(want, y, y.abs() * (SUM + P.HALF_ULP[torch.bfloat16]))


def test_no_rows():
    out, scales, total = B.rms_norm(torch.zeros(0, 64, device=DEV), torch.ones(64, device=DEV), residual=torch.zeros(0, 64, device=DEV), out_dtype="i8")
    assert out.shape == (0, 64) and scales.shape == (0,) and total.shape == (0, 64)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cols", [8, 100, 4096, 20000])
def test_rows_near_the_least_numbers_in_eight_bits(cols, dtype):
    """Down to the least number of binary32, where 127 / max|y| is more than 32 bits hold: the symbols are round(y / s) all the same."""
    x, _, w = _inputs(7, cols, torch.float32)
    sizes = torch.tensor([1e-36, 1e-37, 2e-38, 1e-39, 1e-41, 1e-43, 3e-45], dtype=torch.float64, device=DEV)
    x = x.double() / x.double().abs().amax(-1, keepdim=True)
    tiny = (x * sizes[:, None]).to(dtype)
    plain = (P.wide(tiny), *B.quantise_rows(tiny), torch.zeros(7, dtype=torch.float64))
    # the same by small weights behind rows of ordinary size
    rows = x.to(dtype)
    by = 1 / torch.sqrt((P.wide(rows) ** 2).mean(-1) + EPS)
    normed = []
    for size in sizes.tolist():
        small = (w.double() * size).to(dtype)
        q, s, _ = B.rms_norm(rows, small, EPS, out_dtype="i8")
        normed.append((P.rms_norm(rows, small, EPS, None)[0], q, s, by * 2.0 ** -150))
    for y, q, s, product in (plain, *normed):
        most = y.abs().amax(-1)
        # s is rounded to a multiple of 2^-149, and 127 of it may miss the row's largest by 127 halves of that; so is the product with a weight before
        P.assert_within(s, most / 127, (most * SUM + product) / 127 + 2.0 ** -150)
        bound = P.wide(s)[:, None] * (0.5 + 2.0 ** -12) + y.abs() * SUM + 127 * 2.0 ** -150
        assert ((P.wide(q) * P.wide(s)[:, None] - y).abs() <= torch.maximum(bound, torch.where(P.wide(s) == 0, most, 0.0)[:, None])).all()
        assert (q[s == 0] == 0).all() and (q >= -127).all()
        assert ((q.cpu() > 0) <= (y > 0)).all() and ((q.cpu() < 0) <= (y < 0)).all()


@pytest.mark.parametrize("rows,cols", [((1 << 26) + 3, 8), ((1 << 24) + 1, 1032)])
def test_rows_beyond_one_dimension_of_a_launch(rows, cols):
    """More rows than 2^32 threads have: every row is written."""
    some = torch.randn(4096, cols, device=DEV).to(torch.bfloat16)
    x = some[:1].expand(rows, cols) if cols > 64 else some.repeat(rows // 4096 + 1, 1)[:rows]
    q, scales = B.quantise_rows(x)
    want, by = B.quantise_rows(some)
    torch.cuda.synchronize()
    for at in (0, 1, rows // 2, (1 << 22) - 1, 1 << 22, 1 << 24, rows - 1):
        i = 0 if cols > 64 else at % 4096
        assert torch.equal(q[at], want[i]) and torch.equal(scales[at], by[i]), at
    if cols > 64:
        assert torch.equal(scales, by[:1].expand(rows))
    else:
        assert torch.equal(scales[:rows // 4096 * 4096].view(-1, 4096), by.expand(rows // 4096, 4096))


@pytest.mark.parametrize("cols", [64, 4096, 20000])
def test_rows_that_pass_the_largest_number_behind_the_norm(cols):
    """Rows and weights are numbers, their product behind the norm is not: no scale, no symbols; one beside them has its own."""
    x = torch.full((3, cols), 0.5, device=DEV)
    x[1] = 2.0 ** -30
    w = torch.full((cols,), 3e38, device=DEV)
    q, s, _ = B.rms_norm(x, w, 1e-5, out_dtype="i8")
    assert torch.isfinite(s).tolist() == [True, True, True] and (q == 127).all()
    x[2, 1:] = 0                                                       # its norm is sqrt(cols) / 0.5
    q, s, _ = B.rms_norm(x, w, 1e-5, out_dtype="i8")
    assert torch.isnan(s).tolist() == [False, False, True] and (q[:2] == 127).all() and (q[2] == 0).all()
