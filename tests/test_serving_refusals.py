"""What the operators of a serving step (place_tokens, embed, adapt, sample) refuse: the library by an error code before anything is enqueued (no GPU needed), the binding by a
ValueError before the library is called."""
import ctypes as C

import pytest
import torch

from paper_2406_06237_amd import binding as B

E_NULL, E_RANGE = -1, -2
FAR = 1 << 30                                          # addresses are never followed: every call here is refused first, or has nothing to do
BF16 = torch.bfloat16


def _args(kind, first, change):
    """Every pointer of its own, far from all others."""
    a = kind()
    at = 1 << 32
    for name, field in kind._fields_:
        if field is C.c_void_p:
            setattr(a, name, at)
            at += FAR
    for name, value in {**first, **change}.items():
        setattr(a, name, value)
    return a


PLACE = dict(n_seqs=4, n_tokens=8, free_room=20, table_width=4, page_size=16, workspace_bytes=1 << 20)
EMBED = dict(n_tokens=3, vocabulary=10, weight_stride=64, out_stride=64, cols=64, weight_dtype=B.OUT_U8, out_dtype=B.OUT_BF16, scale=1.0)
ADAPT = dict(rows=4, cols=64, x_stride=32, a_stride=256, a_row_stride=32, b_stride=512, b_row_stride=8, base_stride=64, mul_stride=64, residual_stride=64, out_stride=64,
             adapters=3, k=32, rank=8, x_dtype=B.I8, base_dtype=B.OUT_BF16, out_dtype=B.OUT_BF16, workspace_bytes=1 << 28)
SAMPLE = dict(rows=2, logits_stride=100, vocabulary=100, dtype=B.OUT_F32, temperature=1.0, top_p=1.0)


def _place(**change):
    a = _args(B.PlaceArgs, PLACE, change)                # (lives until the call is done)
    return B.lib().anszp_place(C.addressof(a), None)


def _embed(**change):
    a = _args(B.EmbedArgs, EMBED, change)                # (lives until the call is done)
    return B.lib().anszp_embed(C.addressof(a), None)


def _adapt(**change):
    a = _args(B.AdaptArgs, ADAPT, change)                # (lives until the call is done)
    return B.lib().anszp_adapt(C.addressof(a), None)


def _sample(**change):
    a = _args(B.SampleArgs, SAMPLE, change)                # (lives until the call is done)
    return B.lib().anszp_sample(C.addressof(a), None)


@pytest.mark.parametrize("change,code", [
    *[({n: None}, E_NULL) for n in ("pages", "lengths", "lengths_out", "new_tokens", "free_pages", "n_free", "n_free_out", "slots", "starts", "workspace")],
    (dict(page_size=8), E_RANGE), (dict(page_size=48), E_RANGE), (dict(page_size=1 << 17), E_RANGE), (dict(page_size=0), E_RANGE), (dict(table_width=0), E_RANGE),
    (dict(table_width=(1 << 26) + 1), E_RANGE), (dict(n_seqs=1 << 24), E_RANGE), (dict(n_tokens=1 << 31), E_RANGE), (dict(free_room=1 << 31), E_RANGE),
    (dict(workspace_bytes=79), E_RANGE), (dict(workspace=(1 << 32) + 4), E_RANGE)])
def test_place(change, code):
    assert _place(**change) == code
    assert B.lib().anszp_place(None, None) == E_NULL and B.lib().anszp_place_workspace_bytes(None) == 0


@pytest.mark.parametrize("out", ["pages", "free_pages", "slots", "owners", "starts", "workspace", "lengths_out", "n_free_out"])
@pytest.mark.parametrize("other", ["pages", "free_pages", "slots", "owners", "starts", "workspace", "lengths_out", "n_free_out", "lengths", "n_free", "new_tokens", "ends"])
def test_what_place_writes_meets_nothing(out, other):
    """Apart from lengths and n_free, which may be their own outputs, entry for entry."""
    if out == other or (out, other) in (("lengths_out", "lengths"), ("n_free_out", "n_free")):
        return
    a = _args(B.PlaceArgs, PLACE, {})
    setattr(a, out, getattr(a, other))
    assert B.lib().anszp_place(C.addressof(a), None) == E_RANGE
    a = _args(B.PlaceArgs, PLACE, {})
    a.lengths_out = a.lengths + 4
    assert B.lib().anszp_place(C.addressof(a), None) == E_RANGE


@pytest.mark.parametrize("other", ["pages", "free_pages", "slots", "owners", "starts", "workspace", "lengths_out", "n_free_out", "lengths", "n_free", "new_tokens", "ends"])
def test_what_place_writes_of_last_tokens_meets_nothing(other):
    a = _args(B.PlaceArgs, PLACE, {})
    a.last = getattr(a, other)
    assert B.lib().anszp_place(C.addressof(a), None) == E_RANGE


def test_place_workspace():
    def need(**change):
        a = _args(B.PlaceArgs, PLACE, change)
        return B.lib().anszp_place_workspace_bytes(C.addressof(a))

    assert need(ends=None) == 0 and need() == 80 and need(n_tokens=1 << 20, n_seqs=1000) == 20000 and need(page_size=3) == 0


@pytest.mark.parametrize("change,code", [
    (dict(tokens=None), E_NULL), (dict(weight=None), E_NULL), (dict(out=None), E_NULL), (dict(cols=0), E_RANGE), (dict(cols=1 << 31), E_RANGE), (dict(n_tokens=1 << 31), E_RANGE),
    (dict(vocabulary=1 << 31), E_RANGE), (dict(weight_dtype=B.OUT_F32), E_RANGE), (dict(weight_dtype=B.I8), E_RANGE), (dict(out_dtype=B.OUT_U8), E_RANGE), (dict(zero_point=256), E_RANGE),
    (dict(weight_dtype=B.OUT_BF16), E_RANGE), (dict(weight_dtype=B.OUT_BF16, row_scales=None, zero_point=1), E_RANGE), (dict(out_stride=63), E_RANGE), (dict(n_tokens=0, tokens=None), 0)])
def test_embed(change, code):
    assert _embed(**change) == code
    assert B.lib().anszp_embed(None, None) == E_NULL


@pytest.mark.parametrize("other", ["tokens", "weight", "row_scales"])
def test_embed_over_its_operands(other):
    a = _args(B.EmbedArgs, EMBED, {})
    a.out = getattr(a, other) + 4
    assert B.lib().anszp_embed(C.addressof(a), None) == E_RANGE


@pytest.mark.parametrize("change,code", [
    *[({n: None}, E_NULL) for n in ("x", "a", "b", "ids", "base", "out", "workspace")],
    (dict(rows=1 << 28), E_RANGE), (dict(cols=1 << 31), E_RANGE), (dict(k=0), E_RANGE), (dict(k=(1 << 30) + 1), E_RANGE), (dict(rank=0), E_RANGE), (dict(rank=129), E_RANGE),
    (dict(adapters=1 << 24), E_RANGE), (dict(x_dtype=B.OUT_F32), E_RANGE), (dict(x_dtype=B.OUT_U8), E_RANGE), (dict(base_dtype=B.I8), E_RANGE), (dict(out_dtype=B.OUT_U8), E_RANGE),
    (dict(activation=4), E_RANGE), (dict(out_stride=63), E_RANGE), (dict(workspace_bytes=16), E_RANGE), (dict(workspace=(1 << 32) + 8), E_RANGE),
    (dict(rows=1 << 27, cols=1 << 10, out_stride=1 << 10, x=1 << 60, base=1 << 59, mul=None, residual=None), E_RANGE), (dict(rows=(1 << 28) - 1, cols=8, rank=128, x=1 << 60, base=1 << 59, ids=1 << 58, mul=None, residual=None, x_scales=None), E_RANGE),
    (dict(rows=0, x=None), 0), (dict(cols=0, b=None), 0)])
def test_adapt(change, code):
    assert _adapt(**change) == code
    assert B.lib().anszp_adapt(None, None) == E_NULL and B.lib().anszp_adapt_workspace_bytes(None) == 0


@pytest.mark.parametrize("other,by", [("x", 4), ("a", 4), ("b", 6), ("ids", 0), ("x_scales", 0), ("scales", 4), ("base", 2), ("mul", 128), ("residual", -2)])
def test_adapt_over_its_operands(other, by):
    a = _args(B.AdaptArgs, ADAPT, {})
    a.out = getattr(a, other) + by
    assert B.lib().anszp_adapt(C.addressof(a), None) == E_RANGE


@pytest.mark.parametrize("change", [dict(rows=1 << 26, rank=128, k=4, a_row_stride=0), dict(rows=1 << 15, cols=1 << 17, rank=4, b_row_stride=0, base_stride=1 << 17, out_stride=1 << 17)])
def test_adapt_of_operands_of_a_few_bytes_by_more_threads_than_one_launch_has(change):
    """A thread an element: 2^33 of h, 2^32 of the output."""
    apart = dict(adapters=1, workspace_bytes=1 << 50, x=1 << 60, base=1 << 59, ids=1 << 58, out=1 << 57, mul=None, residual=None, x_scales=None, scales=None)
    assert _adapt(**{**apart, **change}) == E_RANGE


@pytest.mark.parametrize("change", [dict(rows=65537, cols=65535, rank=4, b_row_stride=0, base_stride=65535, out_stride=65535), dict(rows=33818640, rank=127, k=4, a_row_stride=0)])
def test_adapt_where_whole_workgroups_are_the_thread_too_many(change):
    """2^32 - 1 elements of the output and 2^32 - 16 of h, a thread each, are 2^32 threads in workgroups of 256, which one launch has not."""
    apart = dict(adapters=1, workspace_bytes=1 << 50, x=1 << 60, base=1 << 59, ids=1 << 58, out=1 << 57, mul=None, residual=None, x_scales=None, scales=None)
    assert _adapt(**{**apart, **change}) == E_RANGE


def test_adapt_over_a_base_of_another_type_or_stride():
    for change in (dict(base_dtype=B.OUT_F32), dict(base_stride=80)):
        a = _args(B.AdaptArgs, ADAPT, change)
        a.out = a.base
        assert B.lib().anszp_adapt(C.addressof(a), None) == E_RANGE


@pytest.mark.parametrize("change,code", [
    (dict(logits=None), E_NULL), (dict(uniforms=None), E_NULL), (dict(tokens=None), E_NULL), (dict(vocabulary=0), E_RANGE), (dict(vocabulary=(1 << 24) + 1), E_RANGE),
    (dict(rows=1 << 31), E_RANGE), (dict(dtype=B.I8), E_RANGE), (dict(temperatures=None, temperature=-1.0), E_RANGE), (dict(temperatures=None, temperature=float("nan")), E_RANGE),
    (dict(top_ks=None, top_k=-1), E_RANGE), (dict(top_ps=None, top_p=-0.1), E_RANGE), (dict(min_ps=None, min_p=float("nan")), E_RANGE), (dict(rows=0, logits=None), 0)])
def test_sample(change, code):
    assert _sample(**change) == code
    assert B.lib().anszp_sample(None, None) == E_NULL


@pytest.mark.parametrize("out", ["tokens", "chances"])
@pytest.mark.parametrize("other", ["logits", "uniforms", "temperatures", "top_ks", "top_ps", "min_ps", "tokens", "chances"])
def test_sample_over_its_operands(out, other):
    if out == other:
        return
    a = _args(B.SampleArgs, SAMPLE, {})
    setattr(a, out, getattr(a, other))
    assert B.lib().anszp_sample(C.addressof(a), None) == E_RANGE


# ------------------------------------------------------------------------------------------------ the binding
@pytest.fixture
def calls(monkeypatch):
    """The binding with host tensors taken for a GPU's and the library's device calls only counted."""
    seen, real = [], B.lib()

    class Stub:
        def __getattr__(self, name):
            if name.endswith("workspace_bytes"):
                return getattr(real, name)
            return lambda *args: seen.append(name) or 0

    stub = Stub()
    monkeypatch.setattr(B, "lib", lambda: stub)
    monkeypatch.setattr(B, "_torch_with_gpu", torch)
    monkeypatch.setattr(B, "_host", False)
    monkeypatch.setattr(B, "_device_index", lambda torch_, device: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0, raising=False)
    return seen


def _ints(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def _operands():
    return {
        "place": (B.place_tokens, dict(pages=_ints(3, 4), page_size=16, lengths=_ints(3), new=_ints(3), free=_ints(9), n_free=_ints(1), n_tokens=5, ends=_ints(3), status=_ints(2))),
        "embed": (B.embed, dict(tokens=torch.zeros(4, dtype=torch.int64), weight=torch.zeros(9, 32, dtype=torch.uint8), zero_point=3, row_scales=torch.ones(9), status=_ints(2))),
        "adapt": (B.adapt, dict(base=torch.zeros(3, 32), x=torch.zeros(3, 16, dtype=torch.int8), a=torch.zeros(2, 8, 16, dtype=BF16), b=torch.zeros(2, 32, 8, dtype=BF16), ids=_ints(3),
                                x_scales=torch.ones(3), scales=torch.ones(2), mul=torch.zeros(3, 32, dtype=BF16), residual=torch.zeros(3, 32, dtype=BF16), status=_ints(2))),
        "sample": (B.sample, dict(logits=torch.zeros(3, 32), uniforms=torch.zeros(3), temperature=torch.ones(3), top_k=_ints(3), top_p=0.9, min_p=0)),
    }


def test_operands_as_they_should_be(calls):
    for function, operands in _operands().values():
        function(**operands)
    assert calls == ["anszp_place", "anszp_embed", "anszp_adapt", "anszp_sample"]


@pytest.mark.parametrize("which,change", [
    *[("place", {n: None}) for n in ("lengths", "new", "free", "n_free")], ("place", dict(pages=torch.zeros(3, 4, dtype=torch.int64))), ("place", dict(pages=_ints(3, 8)[:, :4])),
    ("place", dict(lengths=_ints(2))), ("place", dict(lengths=_ints(6)[::2])), ("place", dict(new=torch.zeros(3, dtype=torch.int64))), ("place", dict(ends=torch.zeros(3, dtype=torch.bool))),
    ("place", dict(n_free=_ints(2))), ("place", dict(n_tokens=-1)), ("place", dict(n_tokens=1 << 31)), ("place", dict(page_size=-16)), ("place", dict(page_size=1 << 32)),
    ("place", dict(lengths_out=_ints(4))), ("place", dict(n_free_out=torch.zeros(1))), ("place", dict(status=_ints(1))),
    ("embed", dict(weight=None)), ("embed", dict(tokens=_ints(4))), ("embed", dict(tokens=torch.zeros(4, 1, dtype=torch.int64))), ("embed", dict(weight=torch.zeros(9, 32))),
    ("embed", dict(weight=torch.zeros(32, 9, dtype=torch.uint8).t())), ("embed", dict(weight=torch.zeros(9, 32, dtype=BF16))), ("embed", dict(weight=torch.zeros(9, 32, dtype=BF16), zero_point=0)),
    ("embed", dict(zero_point=256)), ("embed", dict(zero_point=-1)), ("embed", dict(row_scales=torch.ones(8))), ("embed", dict(out_dtype="i8")), ("embed", dict(out=torch.zeros(4, 31))),
    ("embed", dict(out=torch.zeros(4, 32, dtype=torch.float16))), ("embed", dict(out=torch.zeros(4, 32), out_dtype="i8")), ("embed", dict(status=_ints(3))),
    *[("adapt", {n: None}) for n in ("x", "a", "b", "ids")], ("adapt", dict(base=torch.zeros(3, 32, dtype=torch.float16))), ("adapt", dict(x=torch.zeros(3, 16))),
    ("adapt", dict(x=torch.zeros(2, 16, dtype=BF16))), ("adapt", dict(a=torch.zeros(2, 8, 15, dtype=BF16))), ("adapt", dict(b=torch.zeros(2, 31, 8, dtype=BF16))),
    ("adapt", dict(b=torch.zeros(3, 32, 8, dtype=BF16))), ("adapt", dict(b=torch.zeros(2, 8, 32, dtype=BF16).transpose(1, 2))), ("adapt", dict(ids=torch.zeros(3, dtype=torch.int64))),
    ("adapt", dict(ids=_ints(4))), ("adapt", dict(x_scales=torch.ones(2))), ("adapt", dict(scales=torch.ones(3))), ("adapt", dict(mul=torch.zeros(3, 32))),
    ("adapt", dict(residual=torch.zeros(3, 31, dtype=BF16))), ("adapt", dict(activation="tanh")), ("adapt", dict(out_dtype="i8")), ("adapt", dict(out=torch.zeros(3, 33, dtype=BF16))),
    ("adapt", dict(status=torch.zeros(2))),
    ("sample", dict(uniforms=None)), ("sample", dict(logits=torch.zeros(3, 32, dtype=torch.float16))), ("sample", dict(logits=torch.zeros(32, 3).t())), ("sample", dict(logits=torch.zeros(32))),
    ("sample", dict(uniforms=torch.zeros(4))), ("sample", dict(uniforms=torch.zeros(3, dtype=torch.float64))), ("sample", dict(temperature=torch.ones(2))), ("sample", dict(temperature=-0.5)),
    ("sample", dict(temperature=float("nan"))), ("sample", dict(top_k=-1)), ("sample", dict(top_k=2.5)), ("sample", dict(top_k=1 << 31)), ("sample", dict(top_k=torch.zeros(3))),
    ("sample", dict(top_p=-1)), ("sample", dict(min_p=torch.zeros(3, dtype=BF16))), ("sample", dict(out=_ints(3))),
])
def test_operands_that_are_refused(calls, which, change):
    function, operands = _operands()[which]
    with pytest.raises(ValueError):
        function(**{**operands, **change})
    assert calls == []


@pytest.mark.parametrize("which", ["place", "embed", "adapt", "sample"])
def test_memory_that_is_no_gpus(monkeypatch, which):
    monkeypatch.setattr(B, "_torch_with_gpu", torch)
    function, operands = _operands()[which]
    with pytest.raises(ValueError, match="Expected a cuda device"):
        function(**operands)


def test_sizes_of_32_bits_and_more(calls):
    """The library's sizes are words of 32 bits: longer ones are refused, not cut.  (Tensors without memory: nothing here is read.)"""
    on = lambda *shape, dtype=torch.int32: torch.empty(shape, dtype=dtype, device="meta")  # noqa: E731
    long = (1 << 32) + 64
    for call in (lambda: B.place_tokens(on(1, long), 16, on(1), on(1), on(3), on(1), 1), lambda: B.embed(on(1, dtype=torch.int64), on(1, long, dtype=torch.uint8)),
                 lambda: B.adapt(on(1, 8, dtype=BF16), on(1, long, dtype=BF16), on(1, 4, long, dtype=BF16), on(1, 8, 4, dtype=BF16), on(1)),
                 lambda: B.adapt(on(1, 8, dtype=BF16), on(1, 4, dtype=BF16), on(1, long, 4, dtype=BF16), on(1, 8, long, dtype=BF16), on(1)),
                 lambda: B.adapt(on(1, 8, dtype=BF16), on(1, 4, dtype=BF16), on(long, 2, 4, dtype=BF16), on(long, 8, 2, dtype=BF16), on(1)),
                 lambda: B.sample(on(1, long, dtype=BF16), on(1, dtype=torch.float32))):
        with pytest.raises(ValueError, match="32 bits"):
            call()
    assert calls == []


@pytest.mark.parametrize("last", [_ints(2), _ints(6)[::2], torch.zeros(3, dtype=torch.int64)])
def test_last_tokens_that_are_refused(calls, last):
    function, operands = _operands()["place"]
    with pytest.raises(ValueError, match="last"):
        function(**operands, last=last)
    assert calls == []
