"""GPU: the operators through the binding's native calls and through its Python path: the same results, the same refusals."""
import pytest
import torch

from paper_2406_06237_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


def _everything():
    g = torch.Generator(device=DEV).manual_seed(3)
    rnd = lambda *s: torch.randn(*s, device=DEV, generator=g)  # noqa: E731
    x, r, w = rnd(9, 512).to(BF16), rnd(9, 512).to(BF16), rnd(512)
    out = [*B.rms_norm(x, w, 1e-5, residual=r, out_dtype="i8"), *B.rms_norm(x, w.to(BF16), out_dtype="f32")[:1], *B.quantise_rows(x)]
    symbols = torch.randint(0, 16, (96, 512), device=DEV, generator=g).to(torch.uint8)
    out.append(B.linear(out[0], symbols, x_scales=out[1], zero_point=7, scale=0.5, channel_scales=rnd(96), bias=rnd(96), activation="gelu", mul=rnd(9, 96), out_dtype="f32"))
    out.append(B.linear(x, r, residual=rnd(9, 9).to(BF16), activation="relu"))
    into = torch.zeros(9, 20, dtype=BF16, device=DEV)
    B.linear(x, r, out=into[:, 3:12])
    out.append(into)
    cache = B.new_kv_cache(4, 16, 2, 64, 4)
    slots = torch.arange(3, 12, device=DEV)
    B.cache_write(cache, x.view(9, 4, 2, 64)[:, 1], r.view(9, 4, 2, 64)[:, 3], slots)
    out += [*B.cache_read(cache, slots, "f32"), *B.cache_read(cache, slots)]
    pages = torch.tensor([[0, 1], [3, 0]], dtype=torch.int32, device=DEV)
    lengths, starts = torch.tensor([12, 9], dtype=torch.int32, device=DEV), torch.tensor([0, 2, 9], dtype=torch.int32, device=DEV)
    q = x.view(9, 8, 64)[:, :6]
    out += [B.attend(q, cache, pages, lengths, starts), B.attend(q, cache, pages, lengths, starts, scale=0.3, out_dtype="f32")]
    into = torch.zeros(9, 8, 64, device=DEV)
    B.attend(q, cache, pages, lengths, starts, out=into[:, 2:])
    return out + [into]


def test_both_paths_give_the_same(monkeypatch):
    assert B._operator_calls()
    native = _everything()
    monkeypatch.setattr(B, "_host", False)
    plain = _everything()
    assert len(native) == len(plain)
    for a, b in zip(native, plain):
        assert (a is None and b is None) or (a.dtype == b.dtype and a.shape == b.shape and torch.equal(a, b))


@pytest.mark.parametrize("native", [True, False])
def test_both_paths_refuse_the_same(monkeypatch, native):
    if not native:
        monkeypatch.setattr(B, "_host", False)
    x, w = torch.zeros(3, 64, dtype=BF16, device=DEV), torch.zeros(32, 64, dtype=BF16, device=DEV)
    cache = B.new_kv_cache(2, 16, 2, 64)
    odd = B.KvCache(*[torch.zeros(2, 2, 12, n, dtype=t, device=DEV) for _ in range(2) for n, t in ((64, torch.uint8), (2, torch.float32))])
    ints = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)  # noqa: E731
    for call in (lambda: B.rms_norm(x, w[0, :63]), lambda: B.rms_norm(x, w[0].cpu()), lambda: B.rms_norm(x, w[0], residual=x.float()), lambda: B.rms_norm(x, None),
                 lambda: B.linear(x, w.cpu()), lambda: B.linear(x, w[:, :32]), lambda: B.linear(x, w, zero_point=3), lambda: B.linear(x, w, activation="exp"),
                 lambda: B.linear(x, w, mul=x), lambda: B.linear(x.float(), w), lambda: B.cache_read(cache, ints(3)),
                 lambda: B.cache_write(cache, x.view(3, 1, 64), x.view(3, 1, 64), torch.zeros(3, dtype=torch.int64, device=DEV)),
                 lambda: B.attend(x.view(3, 1, 64), cache, ints(1, 2), ints(1), ints(2)), lambda: B.attend(x.expand(2, 3, 64)[:, :2], cache, ints(1, 2), ints(2), ints(2))):
        with pytest.raises((ValueError, AttributeError)):
            call()
    for call in (lambda: B.cache_read(odd, torch.zeros(1, dtype=torch.int64, device=DEV)), lambda: B.rms_norm(x[:, :0], w[0, :0]), lambda: B.linear(x[:, :0], w[:, :0])):
        with pytest.raises(B.AnszpError, match="out of range"):
            call()
