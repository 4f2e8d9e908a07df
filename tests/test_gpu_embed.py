"""GPU: tokens looked up as rows, equal to the formula in 32 bits operation by operation."""
import pytest
import torch

import serving_plain as P
from paper_2406_06237_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("n,vocabulary,cols,gap", [(1, 1, 1, 0), (3, 10, 15, 1), (5, 7, 16, 0), (17, 300, 17, 3), (16, 1000, 4096, 0), (2, 50, 8191, 5), (300, 40, 64, 0)])
def test_rows(n, vocabulary, cols, gap, out):
    g = torch.Generator(device=DEV).manual_seed(n + cols)
    tokens = torch.randint(0, vocabulary, (n,), device=DEV, generator=g)
    tokens[n // 2] = -1
    symbols = torch.randint(0, 256, (vocabulary, cols + gap), device=DEV, generator=g).to(torch.uint8)[:, gap:]
    scales = torch.randn(vocabulary, device=DEV, generator=g)
    values = torch.randn(vocabulary, cols + gap, device=DEV, generator=g).to(torch.bfloat16)[:, gap:]
    rounded = lambda t: t.to(torch.bfloat16) if out == "bf16" else t  # noqa: E731
    for weight, more in ((symbols, dict(zero_point=131, row_scales=scales, scale=1.7)), (symbols, dict(zero_point=255)), (values, dict(scale=64.0)), (values, dict(scale=0.3))):
        status = torch.zeros(2, dtype=torch.int32, device=DEV)
        got = B.embed(tokens, weight, out_dtype=out, status=status, **more)
        assert torch.equal(got.cpu(), rounded(P.embed(tokens, weight, **more))) and status.tolist() == [0, 0]
        into = torch.full((n, cols + 2 * gap + 3), 7.0, dtype=got.dtype, device=DEV)
        assert B.embed(tokens, weight, out=into[:, 1:cols + 1], **more).data_ptr() == into[:, 1:].data_ptr()
        assert torch.equal(into[:, 1:cols + 1], got) and (into[:, :1] == 7).all() and (into[:, cols + 1:] == 7).all()


def test_tokens_that_are_not_there():
    weight = torch.ones(5, 40, dtype=torch.bfloat16, device=DEV)
    weight[3] = float("nan")
    status = torch.zeros(2, dtype=torch.int32, device=DEV)
    tokens = torch.tensor([0, 5, -1, 2**40, -2**60, 4], device=DEV)
    got = B.embed(tokens, weight, out_dtype="f32", status=status)
    assert got[:, 0].tolist() == [1, 0, 0, 0, 0, 1] and torch.equal(got[:, :1].expand(-1, 40), got) and status.tolist() == [1, 2]
    assert torch.equal(B.embed(tokens, weight, out_dtype="f32"), got)
    assert torch.isnan(B.embed(torch.tensor([3, 3], device=DEV), weight)).all()
    assert B.embed(tokens[:0], weight).shape == (0, 40)
    assert not B.embed(torch.tensor([-1], device=DEV), weight[:0]).any()


def test_a_table_of_more_than_2_32_symbols():
    """The last rows of 4.3 G symbols."""
    vocabulary, cols = 70000, 61440
    weight = torch.zeros(vocabulary, cols, dtype=torch.uint8, device=DEV)
    weight[-1] = torch.arange(cols, device=DEV) % 251
    weight[0] = 9
    got = B.embed(torch.tensor([vocabulary - 1, 0], device=DEV), weight, out_dtype="f32")
    assert torch.equal(got[0], weight[-1].float()) and (got[1] == 9).all()
