"""What `paper_2605_10793_amd.attention` hands to the library, without a device: tensors that say they lie on one, and a library that notes its calls."""
import struct
import threading

import pytest
import torch

from paper_2605_10793_amd import attention as A, binding

WORKSPACE = 184      # where a packed tree call holds the workspace's address


class Fake:
    """A tensor of zeros that says it lies on GPU `index`."""

    def __init__(self, *shape, dtype=torch.bfloat16, index=0, grad=False):
        self.host = torch.zeros(shape, dtype=dtype)
        self.index, self.requires_grad = index, grad

    def __getattr__(self, name):
        return getattr(self.host, name)

    is_cuda = property(lambda self: self.index >= 0)
    device = property(lambda self: torch.device("cpu"))

    def get_device(self):
        return self.index


class Library:
    """Takes calls as the library would, and asks for a workspace of `size` bytes."""

    def __init__(self, size=4096):
        self.size, self.calls = size, []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, threading.get_ident(), args))
            return binding.OK
        return call

    def conqur_tree_attention_workspace(self, call):
        return self.size

    def conqur_tree_attention(self, call, stream):
        at, size = struct.unpack_from("=QQ", call, WORKSPACE)
        if size < self.size:
            return binding.EINVAL
        self.calls.append(("tree", threading.get_ident(), at))
        return binding.OK


@pytest.fixture
def library(monkeypatch):
    lib = Library()
    monkeypatch.setattr(binding, "load", lambda: lib)
    monkeypatch.setattr(A, "_like", lambda x: None if x is None else Fake(*x.shape, dtype=x.dtype, index=x.index))
    for name, value in (("_cuda_getDevice", lambda: 0), ("_cuda_getCurrentRawStream", lambda i: 0x500 + i), ("_cuda_isCurrentStreamCapturing", lambda: False)):
        monkeypatch.setattr(torch._C, name, value, raising=False)
    return lib


def cache_of(index=0, heads=2, width=64, page=32, pages=4):
    return A.KVCache(Fake(pages, heads, page, width, index=index), Fake(pages, heads, width, page, index=index))


def batch_of(index=0):
    return (Fake(2, dtype=torch.int32, index=index), Fake(1, dtype=torch.int32, index=index), Fake(1, 4, dtype=torch.int32, index=index))


def test_where_the_workspace_is_in_a_call():
    q = Fake(3, 4, 64)
    fields = (*cache_of()._fields, *A._batch(*batch_of()), *A._rows(q, "q", torch.bfloat16, 3, 4, 64), *A._rows(q, "out", torch.bfloat16, 3, 4, 64))
    assert struct.unpack_from("=QQ", A._TREE.pack(*fields, 0, 3, 100, 77, 99, 1, 1.0), WORKSPACE) == (77, 99)


def test_threads_do_not_share_a_workspace(library):
    """Calls of two threads on one stream: what one has enqueued may be followed by the other's first launch before its own second."""
    cache, batch = cache_of(), batch_of()
    met = threading.Barrier(2)

    def serve():
        for _ in range(3):
            met.wait(30)
            A.tree_attention(Fake(3, 4, 64), cache, *batch)
        met.wait(30)           # (a thread's workspaces go with it)

    threads = [threading.Thread(target=serve) for _ in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    rooms = {}
    for _, thread, at in library.calls:
        rooms.setdefault(thread, set()).add(at)
    assert len(rooms) == 2 and len(library.calls) == 6
    a, b = rooms.values()
    assert not a & b


def test_caches_share_a_workspace(library):
    """A model has a cache a layer; their calls on a stream come one behind the other."""
    batch = batch_of()
    for _ in range(3):
        A.tree_attention(Fake(3, 4, 64), cache_of(), *batch)
    assert len({at for _, _, at in library.calls}) == 1
    library.size *= 4                                       # a larger call takes a larger one, which then serves all
    for _ in range(2):
        A.tree_attention(Fake(3, 4, 64), cache_of(), *batch)
    library.size //= 2
    A.tree_attention(Fake(3, 4, 64), cache_of(), *batch)
    assert len({at for _, _, at in library.calls[3:]}) == 1


def test_streams_do_not_share_a_workspace(library, monkeypatch):
    cache, batch = cache_of(), batch_of()
    for stream in (0x100, 0x200):
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i, s=stream: s)
        A.tree_attention(Fake(3, 4, 64), cache, *batch)
    assert len({at for _, _, at in library.calls}) == 2
