"""CPU-only checks of the attention layer's C ABI: struct layouts and refusals that need no device."""
import ctypes
import os
import re

import pytest

from paper_2605_10793_amd import attention as A, binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SIZES = {"void*": 8, "float*": 8, "int64_t*": 8, "int32_t*": 8, "double*": 8, "uint64_t*": 8, "uint64_t": 8, "int64_t": 8, "uint32_t": 4, "float": 4}


def header():
    text = open(os.path.join(ROOT, "include", "conqur.h")).read()
    return re.sub(r"/\*.*?\*/", "", text, flags=re.S)


def fields(name):
    """(C type, field) of a struct of the header, nested structs taken apart."""
    text = header()
    end = text.index("} %s;" % name)
    out = []
    for line in text[text.rindex("typedef struct {", 0, end) + 16:end].split(";"):
        line = " ".join(line.replace("const ", "").split())
        if not line:
            continue
        kind, names = re.match(r"(\w+\*?) (.*)", line).groups()
        for n in names.replace(" ", "").split(","):
            out += [(t, n + "." + f) for t, f in fields(kind)] if kind.startswith("conqur_") else [(kind, n)]
    return out


CODES = {"Q": ("void*", "float*", "int64_t*", "int32_t*", "double*", "uint64_t*", "uint64_t"), "q": ("int64_t",), "I": ("uint32_t",), "f": ("float",)}


@pytest.mark.parametrize("name,form", [("conqur_rotary_call", A._ROTARY), ("conqur_append_call", A._APPEND), ("conqur_tree_call", A._TREE)])
def test_packed_calls_match_the_header(name, form):
    got = form.format.lstrip("=")
    want = fields(name)
    assert len(got) == len(want)
    at = 0
    for code, (kind, field) in zip(got, want):
        assert kind in CODES[code], field
        assert at % SIZES[kind] == 0, field         # C would leave a gap here, the packed form does not
        at += SIZES[kind]
    assert at == form.size and at % 8 == 0


def test_calls_refuse_what_needs_no_device():
    lib = binding.load()
    zero = lambda form: bytes(form.size)  # noqa: E731
    for call in (None, zero(A._ROTARY)):
        assert lib.conqur_rotary(call, None) == binding.EINVAL
        assert lib.conqur_qk_norm_rotary(call, None) == binding.EINVAL
        assert lib.conqur_qk_norm_rotary_backward(call, None, None, None, 0, None) == binding.EINVAL
    for call in (None, zero(A._APPEND)):
        assert lib.conqur_cache_append(call, None) == binding.EINVAL
    for call in (None, zero(A._TREE)):
        assert lib.conqur_tree_attention(call, None) == binding.EINVAL
        assert lib.conqur_tree_attention_workspace(call) == 0
    assert lib.conqur_rotary_frequencies(64, 0, 1e4, 1.0, 0.0, 0.0, 0.0, None, None) == binding.EINVAL


def rotary_call(**change):
    fields_ = dict(q=(0x1000, 256, 128, 2), k=(0, 0, 0, 0), q_out=(0x9000, 256, 128, 2), k_out=(0, 0, 0, 0), q_grad=(0, 0, 0, 0), k_grad=(0, 0, 0, 0),
                   rest=(0, 0, 0x2000, 0x3000), tokens=0, width=128, part=128, layout=0, dtype=1, transposed=0, magnitude=1.0, eps=1e-6)
    fields_.update(change)
    f = fields_
    return A._ROTARY.pack(*f["q"], *f["k"], *f["q_out"], *f["k_out"], *f["q_grad"], *f["k_grad"], *f["rest"], f["tokens"], f["width"], f["part"], f["layout"],
                          f["dtype"], f["transposed"], f["magnitude"], f["eps"], 0)


def test_rotary_arguments():
    """No tokens: nothing is launched, and the scalar arguments are checked all the same."""
    lib = binding.load()
    assert lib.conqur_rotary(rotary_call(), None) == binding.OK
    for bad in (dict(width=127), dict(width=514, part=64), dict(part=0), dict(part=130), dict(part=63), dict(layout=2), dict(dtype=2), dict(transposed=2),
                dict(magnitude=float("inf")), dict(tokens=1 << 31), dict(q=(0x1000, 256, 128, 0)), dict(q=(0x1000, 256, 128, 70000))):
        assert lib.conqur_rotary(rotary_call(**bad), None) == binding.EINVAL, bad
    # with tokens, what is refused before any launch
    for bad in (dict(rest=(0, 0, 0, 0x3000)), dict(rest=(0, 0, 0x2000, 0)), dict(rest=(0, 0, 0x2004, 0x3000)), dict(q=(0x1001, 256, 128, 2)),
                dict(q_out=(0x9000, 256, 64, 2)), dict(q_out=(0x9000, 128, 128, 2)), dict(q_out=(0x9000, 256, 128, 3)), dict(q=(0x1000, -1, 128, 2)),
                dict(q=(0x1000, 1 << 40, 128, 2))):
        assert lib.conqur_rotary(rotary_call(tokens=4, **bad), None) == binding.EINVAL, bad
    assert lib.conqur_qk_norm_rotary(rotary_call(tokens=4), None) == binding.EINVAL          # no weights
    assert lib.conqur_qk_norm_rotary(rotary_call(eps=-1.0), None) == binding.EINVAL


CACHE = dict(k=0x1000, v=0x2000, k_scale=0, v_scale=0, pages=4, heads=2, width=128, page_tokens=64, bits=16)
BATCH = dict(start=0x3000, prefix=0x4000, table=0x5000, stride=8, columns=8, sequences=2)


def tree_call(tokens=4, q=(0x6000, 1024, 128, 8), out=(0x7000, 1024, 128, 8), context=500, workspace=(0x8000, 1 << 40), max_query=4, scale=0.1, **change):
    cache = {k: change.get(k, v) for k, v in CACHE.items()}
    batch = {k: change.get(k, v) for k, v in BATCH.items()}
    return A._TREE.pack(*cache.values(), *batch.values(), *q, *out, change.get("mask", 0), tokens, context, *workspace, max_query, scale)


BAD_CACHES = (dict(k=0), dict(v=0x2008), dict(bits=5), dict(bits=8), dict(bits=8, k_scale=0x100, v_scale=0x104), dict(width=96), dict(page_tokens=8),
              dict(page_tokens=512), dict(page_tokens=48), dict(pages=0), dict(pages=1 << 31), dict(heads=0))
BAD_BATCHES = (dict(start=0), dict(prefix=0x4001), dict(table=0), dict(stride=7), dict(columns=0), dict(sequences=0), dict(sequences=65536))


def test_attention_arguments():
    lib = binding.load()
    assert lib.conqur_tree_attention(tree_call(tokens=0), None) == binding.OK
    size = lib.conqur_tree_attention_workspace(tree_call())
    assert size > 0 and size % 8 == 0
    for bad in BAD_CACHES + BAD_BATCHES + (dict(max_query=0), dict(max_query=65), dict(scale=float("nan")), dict(q=(0x6000, 1024, 128, 7)),
                                           dict(q=(0x6000, 1024, 128, 130), out=(0x7000, 1024, 128, 130)), dict(out=(0x7000, 1024, 128, 4)), dict(context=1 << 31)):
        assert lib.conqur_tree_attention(tree_call(**bad), None) == binding.EINVAL, bad
        assert lib.conqur_tree_attention_workspace(tree_call(**bad)) == 0, bad
    for bad in (dict(q=(0, 1024, 128, 8)), dict(q=(0x6001, 1024, 128, 8)), dict(out=(0x7000, 1024, 64, 8)), dict(mask=0x104), dict(workspace=(0, 1 << 40)),
                dict(workspace=(0x8008, 1 << 40)), dict(workspace=(0x8000, size - 1))):
        assert lib.conqur_tree_attention(tree_call(**bad), None) == binding.EINVAL, bad


def test_append_arguments():
    lib = binding.load()

    def call(tokens=4, k=(0x6000, 256, 128, 2), v=(0x7000, 256, 128, 2), k_values=(0, 0, 0, 0), v_values=(0, 0, 0, 0), **change):
        cache = {n: change.get(n + "_", x) for n, x in CACHE.items()}
        batch = {n: change.get(n + "_", x) for n, x in BATCH.items()}
        return A._APPEND.pack(*cache.values(), *batch.values(), *k, *v, *k_values, *v_values, tokens)

    assert lib.conqur_cache_append(call(tokens=0), None) == binding.OK
    for bad in BAD_CACHES + BAD_BATCHES:
        assert lib.conqur_cache_append(call(**{n + "_": x for n, x in bad.items()}), None) == binding.EINVAL, bad
    for bad in (dict(k=(0, 256, 128, 2)), dict(v=(0x7000, 256, 128, 1)), dict(k_values=(0x9000, 256, 128, 2)), dict(tokens=1 << 31)):
        assert lib.conqur_cache_append(call(**bad), None) == binding.EINVAL, bad


def test_workspace_of_the_gradients():
    assert binding.load().conqur_qk_norm_rotary_workspace(128) % 16 == 0
    assert ctypes.c_uint64(binding.load().conqur_qk_norm_rotary_workspace(1 << 31)).value < 1 << 24
