"""Packed and chunked attention and moves of cached tokens without a device: struct layouts, what the C calls refuse, what the wrappers refuse and hand on."""
import pytest
import torch

from paper_2605_10793_amd import attention as A, binding
from test_attention_cpu import BAD_BATCHES, BAD_CACHES, BATCH, CACHE, CODES, SIZES, fields
from test_attention_calls_cpu import Fake, Library, batch_of, cache_of

I32, F32, I64 = torch.int32, torch.float32, torch.int64


@pytest.mark.parametrize("name,form", [("conqur_attention_call", A._ATTENTION), ("conqur_chunk_call", A._CHUNK), ("conqur_gather_call", A._GATHER)])
def test_packed_calls_match_the_header(name, form):
    got, want, at = form.format.lstrip("="), fields(name), 0
    assert len(got) == len(want)
    for code, (kind, field) in zip(got, want):
        assert kind in CODES[code] and at % SIZES[kind] == 0, field
        at += SIZES[kind]
    assert at == form.size and at % 8 == 0


def test_calls_refuse_what_needs_no_device():
    lib = binding.load()
    for name, form in (("conqur_attention", A._ATTENTION), ("conqur_attention_backward", A._ATTENTION), ("conqur_chunk_attention", A._CHUNK)):
        for call in (None, bytes(form.size)):
            assert getattr(lib, name)(call, None) == binding.EINVAL
            assert getattr(lib, name + "_workspace")(call) == 0
    for call in (None, bytes(A._GATHER.size)):
        assert lib.conqur_cache_gather(call, None) == binding.EINVAL


def attention_call(**change):
    f = dict(q=(0x10000, 1024, 128, 8), k=(0x20000, 256, 128, 2), v=(0x30000, 256, 128, 2), out=(0x40000, 1024, 128, 8), out_grad=(0x50000, 1024, 128, 8),
             q_grad=(0x60000, 1024, 128, 8), k_grad=(0x70000, 256, 128, 2), v_grad=(0x80000, 256, 128, 2), lse=0x90000, start=0xa0000, first=0, last=0, slopes=0,
             tokens=4, sequences=1, width=128, window=0, cap=0.0, scale=0.1, zero_rest=0, workspace=0, bytes=0)
    f.update(change)
    return A._ATTENTION.pack(*(x for v in f.values() for x in (v if isinstance(v, tuple) else (v,))))


def test_attention_arguments():
    lib = binding.load()
    both = (lib.conqur_attention, lib.conqur_attention_backward)
    for call in both:
        assert call(attention_call(tokens=0), None) == binding.OK
    anything = (dict(width=72), dict(width=256), dict(width=0), dict(sequences=0), dict(sequences=65536), dict(cap=-1.0), dict(cap=float("inf")), dict(cap=float("nan")),
                dict(scale=float("nan")), dict(window=1 << 31), dict(tokens=1 << 31), dict(tokens=(1 << 29), q=(0x10000, 1024, 128, 8)), dict(k=(0x20000, 256, 128, 0)),
                dict(k=(0x20000, 256, 128, 3)), dict(q=(0x10000, 1024, 128, 130)))
    for bad in anything:
        for call in both:
            assert call(attention_call(**bad), None) == binding.EINVAL, bad
        assert lib.conqur_attention_workspace(attention_call(**bad)) == lib.conqur_attention_backward_workspace(attention_call(**bad)) == 0
    launch = (dict(q=(0, 1024, 128, 8)), dict(q=(0x10001, 1024, 128, 8)), dict(k=(0x20000, -1, 128, 2)), dict(v=(0x30000, 256, 1 << 40, 2)),
              dict(v=(0x30000, 256, 128, 1)), dict(out=(0x40000, 1024, 128, 4)), dict(start=0), dict(start=0xa0002), dict(first=0x102), dict(last=0x101),
              dict(slopes=0x103), dict(lse=0x102))
    for bad in launch:
        for call in both:
            assert call(attention_call(workspace=0x1000, bytes=1 << 40, **bad), None) == binding.EINVAL, bad
    assert lib.conqur_attention(attention_call(out=(0x40000, 1024, 64, 8)), None) == binding.EINVAL          # overlapping rows
    backward = (dict(lse=0), dict(out_grad=(0, 0, 0, 0)), dict(q_grad=(0x60000, 128, 128, 8)), dict(k_grad=(0x70000, 256, 128, 8)), dict(v_grad=(0, 256, 128, 2)))
    for bad in backward:
        assert lib.conqur_attention_backward(attention_call(workspace=0x1000, bytes=1 << 40, **bad), None) == binding.EINVAL, bad
    need = lib.conqur_attention_backward_workspace(attention_call())
    assert need > 0
    for room in (dict(workspace=0, bytes=1 << 40), dict(workspace=0x1008, bytes=1 << 40), dict(workspace=0x1000, bytes=need - 1)):
        assert lib.conqur_attention_backward(attention_call(**room), None) == binding.EINVAL


@pytest.mark.parametrize("cap,scale,fine", [(4096.0, 0.1, True), (4100.0, 0.1, False), (1e30, 0.1, False), (1e-37, 0.1, True), (1e-40, 0.1, False), (1e-20, 1e20, False),
                                            (0.0, 1e38, True), (0.0, 3e38, False), (50.0, 0.0, True), (50.0, -0.1, True)])
def test_caps_and_scales_that_32_bits_hold(cap, scale, fine):
    """A capped score is off by cap 2^-23, and what is divided by the cap must not overflow."""
    lib = binding.load()
    want = binding.OK if fine else binding.EINVAL
    assert lib.conqur_attention(attention_call(cap=cap, scale=scale, tokens=0), None) == want
    assert lib.conqur_attention_backward(attention_call(cap=cap, scale=scale, tokens=0), None) == want
    assert lib.conqur_chunk_attention(chunk_call(cap=cap, scale=scale, tokens=0), None) == want


def test_workgroups_that_32_bits_count():
    """Sequences times key heads, however few the tokens: a launch holds fewer than 2^32 threads."""
    lib = binding.load()

    def call(sequences, heads, tokens=0):
        return attention_call(sequences=sequences, tokens=tokens, q=(0x10000, heads * 128, 128, heads), k=(0x20000, heads * 128, 128, heads),
                              v=(0x30000, heads * 128, 128, heads), out=(0x40000, heads * 128, 128, heads))
    for sequences, heads, forward, backward in ((65535, 64, True, True), (65535, 200, True, False), (65535, 256, False, False), (1000, 65535, False, False),
                                                (120, 65535, True, True), (250, 65535, True, False)):
        assert lib.conqur_attention(call(sequences, heads), None) == (binding.OK if forward else binding.EINVAL)
        assert lib.conqur_attention_backward(call(sequences, heads), None) == (binding.OK if backward else binding.EINVAL)
        assert bool(lib.conqur_attention_backward_workspace(call(sequences, heads, 1))) == backward


def test_workspace_of_rows_that_are_laid_out():
    """None for rows at multiples of 16 bytes; a copy for each tensor whose are not, or lie far apart."""
    lib = binding.load()
    assert lib.conqur_attention_workspace(attention_call()) == 0
    one = lib.conqur_attention_workspace(attention_call(q=(0x10002, 1024, 128, 8)))
    assert one == 4 * 8 * 128 * 2 == lib.conqur_attention_workspace(attention_call(q=(0x10000, 1028, 128, 8)))
    assert lib.conqur_attention_workspace(attention_call(k=(0x20000, 1 << 22, 128, 2))) == 4 * 2 * 128 * 2
    assert lib.conqur_attention_workspace(attention_call(k=(0x20000, (1 << 22) - 8, 128, 2))) == 0
    assert lib.conqur_attention(attention_call(q=(0x10002, 1024, 128, 8), workspace=0x1000, bytes=one - 1), None) == binding.EINVAL
    plain = lib.conqur_attention_backward_workspace(attention_call())
    assert lib.conqur_attention_backward_workspace(attention_call(out_grad=(0x50002, 1024, 128, 8))) == plain + one


def chunk_call(tokens=4, q=(0x60000, 1024, 128, 8), out=(0x70000, 1024, 128, 8), first=0, last=0, slopes=0, context=500, workspace=(0x8000, 1 << 40), max_query=4, window=0,
               cap=0.0, scale=0.1, **change):
    cache = {k: change.get(k, v) for k, v in CACHE.items()}
    batch = {k: change.get(k, v) for k, v in BATCH.items()}
    return A._CHUNK.pack(*cache.values(), *batch.values(), *q, *out, first, last, slopes, tokens, context, *workspace, max_query, window, cap, scale, 0, 0)


def test_chunk_arguments():
    lib = binding.load()
    assert lib.conqur_chunk_attention(chunk_call(tokens=0), None) == binding.OK
    long = dict(columns=100, stride=100, context=6400)          # (short contexts are not cut into runs, and need no room)
    size = lib.conqur_chunk_attention_workspace(chunk_call(**long))
    assert size > 0 and lib.conqur_chunk_attention_workspace(chunk_call()) == 0
    for bad in BAD_CACHES + BAD_BATCHES + (dict(max_query=0), dict(max_query=1 << 22), dict(scale=float("inf")), dict(cap=-0.5), dict(cap=float("nan")),
                                           dict(window=1 << 31), dict(q=(0x60000, 1024, 128, 7)), dict(out=(0x70000, 1024, 128, 4)), dict(context=1 << 31)):
        assert lib.conqur_chunk_attention(chunk_call(**bad), None) == binding.EINVAL, bad
        assert lib.conqur_chunk_attention_workspace(chunk_call(**bad)) == 0, bad
    for bad in (dict(q=(0, 1024, 128, 8)), dict(out=(0x70000, 1024, 64, 8)), dict(first=0x102), dict(last=0x102), dict(slopes=0x102), dict(workspace=(0, 1 << 40)),
                dict(workspace=(0x8008, 1 << 40)), dict(workspace=(0x8000, size - 1))):
        assert lib.conqur_chunk_attention(chunk_call(**long, **bad), None) == binding.EINVAL, bad


def gather_call(count=4, tokens=0x6000, start=0x7000, table=0x8000, to_table=0x9000, stride=8, to_stride=4, columns=8, to_columns=4, sequences=2, **change):
    cache = {k: change.get(k, v) for k, v in CACHE.items()}
    return A._GATHER.pack(*cache.values(), tokens, start, table, to_table, stride, to_stride, count, columns, to_columns, sequences, 0)


def test_gather_arguments():
    lib = binding.load()
    assert lib.conqur_cache_gather(gather_call(count=0), None) == binding.OK
    for bad in BAD_CACHES + (dict(count=1 << 31), dict(sequences=0), dict(sequences=65536), dict(columns=0), dict(to_columns=0), dict(columns=1 << 31), dict(tokens=0),
                             dict(tokens=0x6002), dict(start=0), dict(table=0), dict(to_table=0x9001), dict(stride=7), dict(to_stride=3), dict(stride=1 << 40),
                             dict(to_stride=-1)):
        assert lib.conqur_cache_gather(gather_call(**bad), None) == binding.EINVAL, bad


# ------------------------------------------------------------------------------------------------ wrappers

@pytest.fixture
def library(monkeypatch):
    class Both(Library):
        def conqur_attention_workspace(self, call):
            return 0

        def conqur_attention_backward_workspace(self, call):
            return 512

        def conqur_chunk_attention_workspace(self, call):
            return 0
    lib = Both()
    monkeypatch.setattr(binding, "load", lambda: lib)
    monkeypatch.setattr(A, "_kept", A._Kept())
    monkeypatch.setattr(A, "_like", lambda x: None if x is None else Fake(*x.shape, dtype=x.dtype, index=x.index))
    for name, value in (("_cuda_getDevice", lambda: 0), ("_cuda_getCurrentRawStream", lambda i: 0x500 + i), ("_cuda_isCurrentStreamCapturing", lambda: False)):
        monkeypatch.setattr(torch._C, name, value, raising=False)
    return lib


def packed_arguments(**change):
    a = dict(q=Fake(3, 4, 64), k=Fake(3, 2, 64), v=Fake(3, 2, 64), start=Fake(2, dtype=I32))
    a.update(change)
    return a


def gradient_arguments(**change):
    return packed_arguments(**{**dict(out=Fake(3, 4, 64), lse=Fake(3, 4, dtype=F32), grad=Fake(3, 4, 64)), **change})


def chunk_arguments(**change):
    start, prefix, table = batch_of()
    return {**dict(q=Fake(3, 4, 64), cache=cache_of(), start=start, prefix=prefix, table=table), **change}


def gather_arguments(**change):
    return {**dict(cache=cache_of(), tokens=Fake(5, dtype=I32), start=Fake(2, dtype=I32), table=Fake(1, 4, dtype=I32), to_table=Fake(1, 4, dtype=I32)), **change}


def test_what_is_called(library):
    A.attention(**packed_arguments())
    A.attention_backward(**gradient_arguments())
    A.chunk_attention(**chunk_arguments())
    A.gather(**gather_arguments())
    assert [name for name, *_ in library.calls] == ["conqur_attention", "conqur_attention_backward", "conqur_chunk_attention", "conqur_cache_gather"]


OPTIONS = dict(first=Fake(3, dtype=I32), last=Fake(3, dtype=I32), slopes=Fake(4, dtype=F32))
BAD_OPTIONS = [dict(first=Fake(4, dtype=I32)), dict(first=Fake(3, dtype=I64)), dict(last=Fake(3, 1, dtype=I32)), dict(slopes=Fake(2, dtype=F32)),
               dict(slopes=Fake(4, dtype=torch.bfloat16)), dict(window=-1), dict(window=1 << 31)]


@pytest.mark.parametrize("call, arguments, bad", [
    *((A.attention, packed_arguments, b) for b in BAD_OPTIONS + [
        dict(k=Fake(4, 2, 64)), dict(k=Fake(3, 2, 32)), dict(v=Fake(3, 1, 64)), dict(q=Fake(3, 64)), dict(q=Fake(3, 4, 64, dtype=F32)), dict(v=Fake(3, 2, 64, dtype=F32)),
        dict(start=Fake(1, dtype=I32)), dict(start=Fake(2, dtype=I64)), dict(start=Fake(2, 2, dtype=I32)), dict(out=Fake(3, 2, 64))]),
    *((A.attention_backward, gradient_arguments, b) for b in BAD_OPTIONS + [
        dict(lse=Fake(3, 2, dtype=F32)), dict(lse=Fake(3, 4)), dict(grad=Fake(3, 4, 32)), dict(grad=Fake(3, 4, 64, dtype=F32)), dict(out=Fake(2, 4, 64))]),
    *((A.chunk_attention, chunk_arguments, b) for b in BAD_OPTIONS + [
        dict(q=Fake(3, 64)), dict(q=Fake(3, 4, 32)), dict(out=Fake(3, 4, 32)), dict(prefix=Fake(2, dtype=I32)), dict(table=Fake(1, 4, dtype=I64))]),
    *((A.gather, gather_arguments, b) for b in [
        dict(tokens=Fake(5, dtype=I64)), dict(tokens=Fake(5, 1, dtype=I32)), dict(start=Fake(1, dtype=I32)), dict(start=Fake(3, dtype=I32)),
        dict(table=Fake(2, 4, dtype=I32)), dict(to_table=Fake(1, 4, dtype=I64)), dict(to_table=Fake(4, dtype=I32))])])
def test_arguments_are_refused(library, call, arguments, bad):
    call(**arguments(**({} if call is A.gather else OPTIONS)))
    library.calls.clear()
    with pytest.raises((ValueError, IndexError)):
        call(**arguments(**bad))
    assert not library.calls


@pytest.mark.parametrize("call, arguments, names", [
    (A.attention, packed_arguments, ("q", "k", "v", "start")), (A.attention_backward, gradient_arguments, ("q", "k", "v", "start", "out", "lse", "grad")),
    (A.chunk_attention, chunk_arguments, ("q", "start", "prefix", "table")), (A.gather, gather_arguments, ("tokens", "start", "table", "to_table"))])
@pytest.mark.parametrize("index", [1, -1])
def test_tensors_of_another_device_are_refused(library, call, arguments, names, index):
    for name in names:
        a = arguments()
        x = a[name]
        a[name] = Fake(*x.shape, dtype=x.dtype, index=index)
        with pytest.raises(ValueError):
            call(**a)
    if call is not A.gather:
        for name, x in OPTIONS.items():
            with pytest.raises(ValueError):
                call(**arguments(**{name: Fake(*x.shape, dtype=x.dtype, index=index)}))
    assert not library.calls


def test_gradients_are_not_lost(library):
    for name in ("q", "k", "v"):
        a = packed_arguments()
        a[name] = Fake(*a[name].shape, grad=True)
        with pytest.raises(ValueError, match="autograd"):
            A.attention(**a)
        with torch.no_grad():
            A.attention(**a)
    with pytest.raises(ValueError, match="autograd"):
        A.chunk_attention(**chunk_arguments(q=Fake(3, 4, 64, grad=True)))


def test_workspace_of_keys_that_are_shared():
    """Few rows with many keys leave their parts of results there: 4 numbers a row and its entries, twice those of the gradients."""
    lib = binding.load()

    def call(tokens, heads, kv, **change):
        return attention_call(tokens=tokens, q=(0x10000, heads * 128, 128, heads), k=(0x20000, kv * 128, 128, kv), v=(0x30000, kv * 128, 128, kv),
                              out=(0x40000, heads * 128, 128, heads), **change)
    rows = (2048 * 2 // 128 + 1 + 2) * 128 * 8          # eight parts of 256 keys
    assert lib.conqur_attention_workspace(call(2048, 2, 1)) == rows * (16 + 128 * 4)
    assert lib.conqur_attention_workspace(call(1200, 2, 1)) == lib.conqur_attention_workspace(call(2048, 2, 1, window=1200)) == 0
    assert lib.conqur_attention_workspace(call(8192, 32, 8)) == 0
    assert lib.conqur_attention(call(2048, 2, 1, workspace=0x1000, bytes=rows * (16 + 128 * 4) - 1), None) == binding.EINVAL
