"""GPU: each kernel of the matrix product at sizes that reach it, from rows that begin at multiples of 16 bytes and from others, with and without a
workspace, against the formula in 64 bits."""
import ctypes as C

import pytest
import torch

import operators_plain as P
from linear_sizes import SIZES
from paper_2406_06237_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
CASES = [(name, *size) for name, sizes in SIZES.items() for size in sizes]


def _inputs(rows, cols, k, eight):
    g = torch.Generator(device=DEV).manual_seed(rows + cols + k)
    rnd = lambda *s: torch.randn(*s, device=DEV, generator=g)  # noqa: E731
    if eight:
        x = torch.randint(-127, 128, (rows, k), device=DEV, generator=g).to(torch.int8)
        w = torch.randint(0, 256, (cols, k), device=DEV, generator=g).to(torch.uint8)
        return dict(x=x, weight=w, x_scales=torch.rand(rows, device=DEV, generator=g) / 64, channel_scales=torch.rand(cols, device=DEV, generator=g) / (64 * k ** 0.5), zero_point=97)
    return dict(x=rnd(rows, k).to(torch.bfloat16), weight=(rnd(cols, k) / k ** 0.5).to(torch.bfloat16))


def _apart(t, pad):
    """The same rows, further apart."""
    rows, k = t.shape
    wide = torch.zeros(rows, -(-k // pad) * pad + pad, dtype=t.dtype, device=t.device)
    wide[:, :k] = t
    return wide[:, :k]


@pytest.mark.parametrize("name,rows,cols,k,eight", CASES)
def test_kernel(name, rows, cols, k, eight):
    print(name, rows, cols, k, eight, flush=True)
    a = _inputs(rows, cols, k, eight)
    want, error = P.linear(a["x"], a["weight"], a.get("x_scales"), a.get("zero_point", 0), 1.0, a.get("channel_scales"))
    got = B.linear(**a, out_dtype="f32")
    P.assert_within(got, want, error + want.abs() * 2.0 ** -23, name)
    near = B.linear(**{**a, "x": _apart(a["x"], 16), "weight": _apart(a["weight"], 16)}, out_dtype="f32")       # whole pieces of 16 bytes
    P.assert_within(near, want, error + want.abs() * 2.0 ** -23, name)
    g = torch.Generator(device=DEV).manual_seed(1)
    bias, mul, residual = torch.randn(cols, device=DEV, generator=g), torch.randn(rows, cols, device=DEV, generator=g), torch.randn(rows, cols, device=DEV, generator=g)
    full = B.linear(**a, bias=bias, mul=mul.bfloat16(), residual=residual.bfloat16(), activation="silu")
    want, error = P.linear(a["x"], a["weight"], a.get("x_scales"), a.get("zero_point", 0), 1.0, a.get("channel_scales"), bias, "silu", mul.bfloat16(), residual.bfloat16())
    P.assert_within(full, want, error + want.abs() * P.HALF_ULP[torch.bfloat16], name)


@pytest.mark.parametrize("name,rows,cols,k,eight", [c for c in CASES if c[0].endswith("shares")])
def test_shares_with_and_without_a_workspace(name, rows, cols, k, eight):
    """Without one the call takes a kernel that needs none; one that is too small is refused; the words behind it stay as they were."""
    a = _inputs(rows, cols, k, eight)
    out = torch.empty(rows, cols, device=DEV)
    args = B.LinearArgs(x=a["x"].data_ptr(), weight=a["weight"].data_ptr(), out=out.data_ptr(), rows=rows, cols=cols, k=k, x_stride=k, weight_stride=k, out_stride=cols,
                        x_dtype=B.I8 if eight else B.OUT_BF16, out_dtype=B.OUT_F32, zero_point=a.get("zero_point", 0), scale=1.0)
    L, stream = B.lib(), torch.cuda.current_stream().cuda_stream
    need = L.anszp_linear_workspace_bytes(C.addressof(args))
    assert need > 0
    want, error = P.linear(a["x"], a["weight"], zero_point=a.get("zero_point", 0))
    assert L.anszp_linear(C.addressof(args), stream) == 0
    P.assert_within(out, want, error + want.abs() * 2.0 ** -23, "without")
    room = torch.full((need // 4 + 64,), 0x5A5A5A5A, dtype=torch.int32, device=DEV)
    args.workspace, args.workspace_bytes = room.data_ptr(), need - 1
    assert L.anszp_linear(C.addressof(args), stream) == -2
    args.workspace_bytes = need
    out.zero_()
    assert L.anszp_linear(C.addressof(args), stream) == 0
    P.assert_within(out, want, error + want.abs() * 2.0 ** -23, "with")
    assert (room[need // 4:] == 0x5A5A5A5A).all()


def test_shares_in_a_graph():
    a = _inputs(64, 512, 4096, False)
    static = torch.empty(64, 512, dtype=torch.bfloat16, device=DEV)
    B.linear(**a, out=static)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.linear(**a, out=static)
    for _ in range(4):
        a["x"].copy_(torch.randn(64, 4096, device=DEV).to(torch.bfloat16))
        static.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(static, B.linear(**a))
