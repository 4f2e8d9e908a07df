"""What the operators beside the decoded weights refuse: the library by an error code before anything is enqueued (no GPU needed), the binding by
a ValueError before the library is called."""
import ctypes as C

import pytest
import torch

from paper_2406_06237_amd import binding as B

E_NULL, E_RANGE = -1, -2
PTR = 1 << 20                                          # never followed: every call here is refused first


def _norm(**change):
    a = B.NormArgs(x=PTR, residual=None, total=None, weight=PTR, out=PTR, out_scales=PTR, rows=4, x_stride=64, out_stride=64, cols=64, dtype=B.OUT_BF16,
                   weight_dtype=B.OUT_BF16, out_dtype=B.I8, normalise=1, eps=1e-6)
    for name, value in change.items():
        setattr(a, name, value)
    return B.lib().anszp_rms_norm(C.addressof(a), None)


@pytest.mark.parametrize("change,code", [
    (dict(x=None), E_NULL), (dict(weight=None), E_NULL), (dict(out=None), E_NULL), (dict(out_scales=None), E_NULL),
    (dict(cols=0), E_RANGE), (dict(cols=1 << 31), E_RANGE), (dict(rows=1 << 31), E_RANGE), (dict(dtype=B.OUT_U8), E_RANGE), (dict(dtype=B.I8), E_RANGE),
    (dict(out_dtype=B.OUT_U8), E_RANGE), (dict(out_dtype=4), E_RANGE), (dict(weight_dtype=B.I8), E_RANGE), (dict(out_stride=63), E_RANGE),
    (dict(total=PTR, total_stride=10), E_RANGE), (dict(rows=0, x=None, out=None), 0)])
def test_norm(change, code):
    assert _norm(**change) == code
    assert B.lib().anszp_rms_norm(None, None) == E_NULL


def _linear(**change):
    a = B.LinearArgs(x=PTR, weight=PTR, out=PTR, rows=4, cols=64, x_stride=64, weight_stride=64, out_stride=64, k=64, x_dtype=B.I8, out_dtype=B.OUT_BF16, scale=1.0)
    for name, value in change.items():
        setattr(a, name, value)
    return B.lib().anszp_linear(C.addressof(a), None)


@pytest.mark.parametrize("change,code", [
    (dict(x=None), E_NULL), (dict(weight=None), E_NULL), (dict(out=None), E_NULL), (dict(k=0), E_RANGE), (dict(k=65537), E_RANGE),
    (dict(k=(1 << 30) + 1, x_dtype=B.OUT_BF16), E_RANGE), (dict(rows=1 << 31), E_RANGE), (dict(cols=1 << 31), E_RANGE), (dict(x_dtype=B.OUT_F32), E_RANGE),
    (dict(x_dtype=B.OUT_U8), E_RANGE), (dict(out_dtype=B.I8), E_RANGE), (dict(zero_point=256), E_RANGE), (dict(activation=4), E_RANGE), (dict(out_stride=60), E_RANGE),
    (dict(rows=0, x=None), 0), (dict(cols=0, weight=None), 0)])
def test_linear(change, code):
    assert _linear(**change) == code
    assert B.lib().anszp_linear(None, None) == E_NULL


def _cache(**change):
    a = B.CacheArg(k=PTR, k_params=PTR, v=PTR, v_params=PTR, n_pages=4, page_size=16, heads=2, head_dim=64, bits=8)
    for name, value in change.items():
        setattr(a, name, value)
    return a


@pytest.mark.parametrize("change,code", [
    (dict(), 0), (dict(bits=2), E_RANGE), (dict(head_dim=96), E_RANGE), (dict(page_size=8), E_RANGE), (dict(page_size=48), E_RANGE), (dict(page_size=1 << 17), E_RANGE),
    (dict(heads=0), E_RANGE), (dict(heads=1 << 16), E_RANGE), (dict(n_pages=1 << 31), E_RANGE), (dict(k=None), E_NULL), (dict(v_params=None), E_NULL),
    (dict(k=PTR + 8), E_RANGE), (dict(v_params=PTR + 4), E_RANGE), (dict(n_pages=0, k=None, v=None, k_params=None, v_params=None), 0)])
def test_cache(change, code):
    a, L = _cache(**change), B.lib()
    assert L.anszp_cache_check(C.addressof(a)) == code
    if code:
        assert L.anszp_cache_write(C.addressof(a), PTR, PTR, B.OUT_F32, 1, 1, 1, 1, PTR, 1, None, None) == code
        assert L.anszp_cache_read(C.addressof(a), PTR, PTR, B.OUT_F32, PTR, 1, None, None) == code


def test_cache_calls():
    a, L = _cache(), B.lib()
    write = lambda k=PTR, v=PTR, dtype=B.OUT_BF16, slots=PTR, n=1, cache=C.addressof(a): L.anszp_cache_write(cache, k, v, dtype, 1, 1, 1, 1, slots, n, None, None)  # noqa: E731
    read = lambda k=PTR, v=PTR, dtype=B.OUT_BF16, slots=PTR, n=1, cache=C.addressof(a): L.anszp_cache_read(cache, k, v, dtype, slots, n, None, None)  # noqa: E731
    for call in (write, read):
        assert call(cache=None) == call(k=None) == call(v=None) == call(slots=None) == E_NULL
        assert call(dtype=B.I8) == call(dtype=B.OUT_U8) == call(n=1 << 31) == E_RANGE
        assert call(n=0, slots=None) == 0


def _attend(cache=None, **change):
    a = B.AttendArgs(q=PTR, out=PTR, pages=PTR, lengths=PTR, starts=PTR, n_tokens=1, n_seqs=1, q_token_stride=128, q_head_stride=64, out_token_stride=128,
                     out_head_stride=64, table_width=4, group=1, out_dtype=B.OUT_BF16, scale=0.1)
    for name, value in change.items():
        setattr(a, name, value)
    a.cache = _cache(**(cache or {}))
    return a


@pytest.mark.parametrize("change,code", [
    (dict(q=None), E_NULL), (dict(out=None), E_NULL), (dict(pages=None), E_NULL), (dict(lengths=None), E_NULL), (dict(starts=None), E_NULL),
    (dict(table_width=0), E_RANGE), (dict(table_width=1 << 27), E_RANGE), (dict(group=0), E_RANGE), (dict(group=257), E_RANGE), (dict(out_dtype=B.I8), E_RANGE),
    (dict(n_tokens=1 << 24), E_RANGE), (dict(n_seqs=1 << 24), E_RANGE), (dict(cache=dict(head_dim=32)), E_RANGE), (dict(cache=dict(v=None)), E_NULL),
    (dict(n_tokens=0, q=None), 0), (dict(n_seqs=0, pages=None), 0)])
def test_attend(change, code):
    a = _attend(**change)
    assert B.lib().anszp_attend(C.addressof(a), None) == code


def test_attend_workspace():
    L = B.lib()
    a = _attend(table_width=4096)
    need = L.anszp_attend_workspace_bytes(C.addressof(a))
    assert need > 0
    a.workspace, a.workspace_bytes = None, need
    assert L.anszp_attend(C.addressof(a), None) == E_NULL
    a.workspace, a.workspace_bytes = PTR, need - 1
    assert L.anszp_attend(C.addressof(a), None) == E_RANGE
    a.workspace, a.workspace_bytes = PTR + 4, need
    assert L.anszp_attend(C.addressof(a), None) == E_RANGE
    for nothing in (_attend(n_tokens=0), _attend(group=0), _attend(table_width=1)):
        assert L.anszp_attend_workspace_bytes(C.addressof(nothing)) == 0
    assert L.anszp_attend_workspace_bytes(None) == 0 and L.anszp_attend(None, None) == E_NULL


# ------------------------------------------------------------------------------------------------ the binding
@pytest.fixture
def calls(monkeypatch):
    """The binding with host tensors taken for a GPU's and the library's device calls only counted."""
    seen, real = [], B.lib()

    class Stub:
        def __getattr__(self, name):
            if name in ("anszp_attend_workspace_bytes", "anszp_linear_workspace_bytes"):
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


BF16 = torch.bfloat16


def _operands():
    cache = B.KvCache(torch.zeros(3, 2, 16, 64, dtype=torch.uint8), torch.zeros(3, 2, 16, 2), torch.zeros(3, 2, 16, 64, dtype=torch.uint8), torch.zeros(3, 2, 16, 2),
                      8, torch.zeros(2, dtype=torch.int32))
    return {
        "norm": (B.rms_norm, dict(x=torch.zeros(3, 64, dtype=BF16), weight=torch.ones(64, dtype=BF16), residual=torch.zeros(3, 64, dtype=BF16))),
        "linear": (B.linear, dict(x=torch.zeros(3, 64, dtype=torch.int8), weight=torch.zeros(32, 64, dtype=torch.uint8), x_scales=torch.ones(3), channel_scales=torch.ones(32),
                                  bias=torch.zeros(32), mul=torch.zeros(3, 32, dtype=BF16), residual=torch.zeros(3, 32, dtype=BF16))),
        "write": (B.cache_write, dict(cache=cache, k=torch.zeros(5, 2, 64), v=torch.zeros(5, 2, 64), slots=torch.zeros(5, dtype=torch.int64))),
        "read": (B.cache_read, dict(cache=cache, slots=torch.zeros(5, dtype=torch.int64))),
        "attend": (B.attend, dict(q=torch.zeros(4, 6, 64, dtype=BF16), cache=cache, pages=torch.zeros(2, 3, dtype=torch.int32), lengths=torch.zeros(2, dtype=torch.int32),
                                  starts=torch.zeros(3, dtype=torch.int32))),
    }


def _cache_with(**change):
    cache = _operands()["read"][1]["cache"]
    for name, value in change.items():
        setattr(cache, name, value)
    return dict(cache=cache)


def test_operands_as_they_should_be(calls):
    for function, operands in _operands().values():
        function(**operands)
    assert calls == ["anszp_rms_norm", "anszp_linear", "anszp_cache_write", "anszp_cache_read", "anszp_attend"]


@pytest.mark.parametrize("which,change", [
    ("norm", dict(x=torch.zeros(3, 64, dtype=torch.float16))), ("norm", dict(x=torch.zeros(64, dtype=BF16))), ("norm", dict(x=torch.zeros(64, 3, dtype=BF16).t())),
    ("norm", dict(weight=torch.ones(63, dtype=BF16))), ("norm", dict(weight=torch.ones(64, dtype=torch.float16))), ("norm", dict(residual=torch.zeros(3, 64))),
    ("norm", dict(residual=torch.zeros(2, 64, dtype=BF16))), ("norm", dict(out_dtype="u8")), ("norm", dict(total=torch.zeros(3, 64))),
    ("linear", dict(x=torch.zeros(3, 64))), ("linear", dict(x=torch.zeros(3, 64, dtype=BF16))), ("linear", dict(weight=torch.zeros(32, 64, dtype=BF16))),
    ("linear", dict(weight=torch.zeros(32, 63, dtype=torch.uint8))), ("linear", dict(weight=torch.zeros(64, 32, dtype=torch.uint8).t())), ("linear", dict(x_scales=torch.ones(4))),
    ("linear", dict(channel_scales=torch.ones(32, dtype=BF16))), ("linear", dict(channel_scales=torch.ones(64)[::2])), ("linear", dict(bias=torch.zeros(32, 1))),
    ("linear", dict(mul=torch.zeros(3, 32))), ("linear", dict(residual=torch.zeros(3, 33, dtype=BF16))), ("linear", dict(activation="tanh")), ("linear", dict(out_dtype="i8")),
    ("linear", dict(zero_point=256)), ("linear", dict(zero_point=-1)), ("linear", dict(out=torch.zeros(3, 31, dtype=BF16))), ("linear", dict(out=torch.zeros(3, 32, dtype=torch.float16))),
    ("linear", dict(x=torch.zeros(3, 64, dtype=BF16), weight=torch.zeros(32, 64, dtype=BF16), zero_point=1)),
    ("write", dict(k=torch.zeros(5, 3, 64))), ("write", dict(v=torch.zeros(5, 2, 64, dtype=BF16))), ("write", dict(v=torch.zeros(4, 2, 64))),
    ("write", dict(slots=torch.zeros(5, dtype=torch.int32))), ("write", dict(slots=torch.zeros(4, dtype=torch.int64))), ("write", dict(k=torch.zeros(5, 64, 2).transpose(1, 2))),
    ("read", dict(slots=torch.zeros(5, 1, dtype=torch.int64))), ("read", dict(out_dtype="i8")), ("read", _cache_with(bits=5)),
    ("read", _cache_with(k=torch.zeros(3, 2, 16, 64))), ("read", _cache_with(v=torch.zeros(2, 2, 16, 64, dtype=torch.uint8))), ("read", _cache_with(k_params=torch.zeros(3, 2, 16, 1))),
    ("read", _cache_with(v_params=torch.zeros(3, 2, 16, 4)[..., ::2])), ("read", _cache_with(status=torch.zeros(1, dtype=torch.int32))),
    ("read", _cache_with(k=torch.zeros(3, 16, 2, 64, dtype=torch.uint8).transpose(1, 2))),
    ("attend", dict(q=torch.zeros(4, 5, 64, dtype=BF16))), ("attend", dict(q=torch.zeros(4, 6, 64))), ("attend", dict(q=torch.zeros(4, 6, 32, dtype=BF16))),
    ("attend", dict(q=torch.zeros(4, 0, 64, dtype=BF16))), ("attend", dict(q=torch.zeros(4, 384, dtype=BF16))), ("attend", dict(pages=torch.zeros(2, 3, dtype=torch.int64))),
    ("attend", dict(pages=torch.zeros(2, 6, dtype=torch.int32)[:, :3])), ("attend", dict(lengths=torch.zeros(3, dtype=torch.int32))), ("attend", dict(starts=torch.zeros(2, dtype=torch.int32))),
    ("attend", dict(out_dtype="i8")), ("attend", dict(out=torch.zeros(4, 6, 32, dtype=BF16))),
])
def test_operands_that_are_refused(calls, which, change):
    function, operands = _operands()[which]
    with pytest.raises(ValueError):
        function(**{**operands, **change})
    assert calls == []


@pytest.mark.parametrize("which", ["norm", "linear", "write", "read", "attend"])
def test_memory_that_is_no_gpus(monkeypatch, which):
    monkeypatch.setattr(B, "_torch_with_gpu", torch)
    function, operands = _operands()[which]
    with pytest.raises(ValueError, match="Expected a cuda device"):
        function(**operands)


def test_new_cache():
    with pytest.MonkeyPatch.context() as m:
        m.setattr(B, "_torch_with_gpu", torch)
        for bad in (dict(bits=3), dict(head_dim=80)):
            with pytest.raises(ValueError):
                B.new_kv_cache(**{**dict(n_pages=2, page_size=16, heads=2, head_dim=64, bits=4, device="cpu"), **bad})
        cache = B.new_kv_cache(2, 16, 3, 128, 4, "cpu")
        assert cache.k.shape == (2, 3, 16, 64) and cache.head_dim == 128 and cache.page_size == 16


def test_page_tables_are_read_row_after_row(calls):
    """Sequence s's pages are entries s * width on: the view of a wider table's first columns is none such, at a width of 1 either; one row of it is."""
    function, operands = _operands()["attend"]
    wide = torch.zeros(2, 6, dtype=torch.int32)
    for width in (1, 2, 5):
        with pytest.raises(ValueError, match="contiguous"):
            function(**{**operands, "pages": wide[:, :width]})
    assert calls == []
    one = dict(q=operands["q"], cache=operands["cache"], lengths=torch.zeros(1, dtype=torch.int32), starts=torch.zeros(2, dtype=torch.int32))
    for pages in (wide[1:, :1], wide[:1, 2:4], torch.zeros(1, 1, dtype=torch.int32)):
        function(pages=pages, **one)
    function(**{**operands, "pages": torch.zeros(2, 1, dtype=torch.int32)})
    assert calls == ["anszp_attend"] * 4


def test_a_page_table_of_no_columns_is_the_librarys_to_refuse(calls):
    """It is out of range, not out of order: its strides say nothing."""
    function, operands = _operands()["attend"]
    function(**{**operands, "pages": torch.zeros(2, 0, dtype=torch.int32)})
    assert calls == ["anszp_attend"]


def test_products_of_more_threads_than_a_launch_has():
    """Refused: a launch would leave them out without an error."""
    for rows, cols in ((1, 1 << 30), (1 << 30, 64), (1 << 20, 1 << 16)):
        assert _linear(rows=rows, cols=cols, k=7, out_stride=cols, x_dtype=B.OUT_BF16) == E_RANGE


def test_attention_of_more_threads_than_a_launch_has():
    """Refused: a launch would leave them out without an error."""
    for cache, many in ((dict(heads=2), dict(n_tokens=(1 << 24) - 1, n_seqs=1, group=256)),                     # 128 rows a workgroup
                        (dict(heads=2, head_dim=256), dict(n_tokens=1 << 23, n_seqs=1, group=256)),
                        (dict(heads=1), dict(n_tokens=64, n_seqs=(1 << 24) - 1, group=1))):                      # 16
        a = _attend(cache=cache, **many)
        assert B.lib().anszp_attend(C.addressof(a), None) == E_RANGE, many


def test_a_norm_without_a_weight_is_refused(calls):
    function, operands = _operands()["norm"]
    with pytest.raises(ValueError, match="weight"):
        function(**{**operands, "weight": None})
    assert calls == []


def test_sizes_of_32_bits_and_more(calls):
    """The library's sizes are words of 32 bits: a longer row, table or page is refused, not cut to what is left of its number.  (Tensors without memory: nothing here is read.)"""
    on = lambda *shape, dtype=BF16: torch.empty(shape, dtype=dtype, device="meta")  # noqa: E731
    long = (1 << 32) + 64
    cache = B.KvCache(on(3, 2, 16, 64, dtype=torch.uint8), on(3, 2, 16, 2, dtype=torch.float32), on(3, 2, 16, 64, dtype=torch.uint8), on(3, 2, 16, 2, dtype=torch.float32))
    tall = B.KvCache(on(1, 2, long, 64, dtype=torch.uint8), on(1, 2, long, 2, dtype=torch.float32), on(1, 2, long, 64, dtype=torch.uint8), on(1, 2, long, 2, dtype=torch.float32))
    wide = B.KvCache(on(1, long, 16, 64, dtype=torch.uint8), on(1, long, 16, 2, dtype=torch.float32), on(1, long, 16, 64, dtype=torch.uint8), on(1, long, 16, 2, dtype=torch.float32))
    ints = lambda *shape: on(*shape, dtype=torch.int32)  # noqa: E731
    for call in (lambda: B.rms_norm(on(1, long), on(long)), lambda: B.quantise_rows(on(1, long)),
                 lambda: B.linear(on(1, long), on(1, long)), lambda: B.linear(on(1, long, dtype=torch.int8), on(1, long, dtype=torch.uint8)),
                 lambda: B.attend(on(1, 2, 64), cache, ints(1, long), ints(1), ints(2)), lambda: B.attend(on(1, 2 * long, 64), cache, ints(1, 1), ints(1), ints(2)),
                 lambda: B.attend(on(1, 2, 64), tall, ints(1, 1), ints(1), ints(2)), lambda: B.attend(on(1, 2 * long, 64), wide, ints(1, 1), ints(1), ints(2)),
                 lambda: B.cache_read(tall, on(1, dtype=torch.int64)), lambda: B.cache_write(wide, on(1, long, 64), on(1, long, 64), on(1, dtype=torch.int64))):
        with pytest.raises(ValueError, match="32 bits"):
            call()
    assert calls == []


FAR = 1 << 30                                          # so far behind PTR that nothing meets


@pytest.mark.parametrize("change", [
    dict(x=PTR), dict(weight=PTR), dict(x=PTR + 4 * 128 - 1), dict(x=PTR - 4 * 64 + 1), dict(weight=PTR + 2), dict(weight=PTR - 64 * 64 + 2),
    dict(mul=PTR + 2, mul_stride=64), dict(residual=PTR + 128, residual_stride=64), dict(residual=PTR, residual_stride=80, out_stride=64),
    dict(out_stride=128, residual=PTR + 100, residual_stride=128), dict(out_stride=128, x=PTR + 256 + 127, x_stride=256), dict(rows=1, x=PTR + 60), dict(cols=1, out_stride=1, weight=PTR + 6)])
def test_products_over_their_operands(change):
    """An output that meets x or the weights, or mul or the residual elsewhere than row for row."""
    assert _linear(**{**dict(x=PTR + FAR, weight=PTR + 2 * FAR), **change}) == E_RANGE


@pytest.mark.parametrize("change", [
    dict(out=PTR), dict(out=PTR + 100), dict(residual=PTR + 3 * FAR, residual_stride=64, out=PTR + 3 * FAR + 511), dict(total=PTR + FAR, total_stride=64),
    dict(total=PTR + 2, total_stride=64), dict(total=PTR, total_stride=70), dict(residual=PTR + 3 * FAR, residual_stride=64, total=PTR + 3 * FAR + 128, total_stride=64)])
def test_norms_over_their_operands(change):
    assert _norm(**{**dict(out=PTR + FAR, weight=PTR + 2 * FAR, out_scales=PTR + 4 * FAR), **change}) == E_RANGE


@pytest.mark.parametrize("change", [dict(n_tokens=2, out_token_stride=0), dict(n_tokens=2, out_token_stride=63), dict(out_head_stride=0), dict(out_head_stride=63),
                                    dict(group=2, cache=dict(heads=1), out_head_stride=0)])
def test_attention_into_rows_over_each_other(change):
    """Rows of the output that share memory would hold one query's result or another's."""
    assert B.lib().anszp_attend(C.addressof(_attend(**change)), None) == E_RANGE


@pytest.mark.parametrize("which,out", [("linear", torch.zeros(3, 32, dtype=BF16)), ("attend", torch.zeros(4, 6, 64, dtype=BF16))])
def test_a_type_that_is_none_beside_an_output(calls, which, out):
    """The output's own type counts, and a name that is no type's is refused all the same."""
    function, operands = _operands()[which]
    for name in ("i8", "fp8", None):
        with pytest.raises(ValueError, match="out_dtype"):
            function(**{**operands, "out": out, "out_dtype": name})
    assert calls == []
