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
    monkeypatch.setattr(A, "_kept", A._Kept())
    monkeypatch.setattr(A, "_like", lambda x: None if x is None else Fake(*x.shape, dtype=x.dtype, index=x.index))
    for name, value in (("_cuda_getDevice", lambda: 0), ("_cuda_getCurrentRawStream", lambda i: 0x500 + i), ("_cuda_isCurrentStreamCapturing", lambda: False)):
        monkeypatch.setattr(torch._C, name, value, raising=False)
    return lib


def cache_of(index=0, heads=2, width=64, page=32, pages=4):
    return A.KVCache(Fake(pages, heads, page, width, index=index), Fake(pages, heads, width, page, index=index))


def batch_of(index=0):
    return (Fake(2, dtype=torch.int32, index=index), Fake(1, dtype=torch.int32, index=index), Fake(1, 4, dtype=torch.int32, index=index))


def test_where_the_workspace_is_in_a_call():
    codes = A._TREE.format.lstrip("=")
    call = A._TREE.pack(*range(1, len(codes) + 1))
    assert struct.unpack_from("=QQ", call, WORKSPACE) == (len(codes) - 3, len(codes) - 2)      # before max_query and scale


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


# ------------------------------------------------------------------------------------------------ devices

def rotary_arguments(index=0):
    return dict(q=Fake(3, 4, 64, index=index), positions=Fake(3, dtype=torch.int64, index=index), k=Fake(3, 2, 64, index=index))


def norm_arguments(index=0):
    return dict(rotary_arguments(index), q_weight=Fake(64, index=index), k_weight=Fake(64, index=index))


def cache_arguments(index=0):
    start, prefix, table = batch_of(index)
    return dict(start=start, prefix=prefix, table=table)


CALLS = {  # what is called, its tensors on a device, and whether it takes a plan or a cache
    "rotary": (rotary_arguments, lambda a, at: A.rotary(a.pop("plan"), **a)),
    "norm": (norm_arguments, lambda a, at: A.qk_norm_rotary(a.pop("plan"), **a)),
    "gradient": (lambda i=0: dict(norm_arguments(i), q_grad=Fake(3, 4, 64, index=i), k_grad=Fake(3, 2, 64, index=i)),
                 lambda a, at: A.qk_norm_rotary_backward(a.pop("plan"), **a)),
    "append": (lambda i=0: dict(cache_arguments(i), k=Fake(3, 2, 64, index=i), v=Fake(3, 2, 64, index=i)), lambda a, at: A.append(cache_of(at), **a)),
    "attention": (lambda i=0: dict(cache_arguments(i), q=Fake(3, 4, 64, index=i), mask=Fake(3, dtype=torch.int64, index=i), out=Fake(3, 4, 64, index=i)),
                  lambda a, at: A.tree_attention(a.pop("q"), cache_of(at), **a)),
}


class Plan:
    def __init__(self, index):
        self.turns, self.part, self.layout, self.magnitude = Fake(32, dtype=torch.float64, index=index), 64, 0, 1.0


@pytest.fixture
def current(monkeypatch, library):
    """The current device, which `torch.cuda.device` changes, its stream and whether that is being captured."""
    at = [0]

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.before, at[0] = at[0], self.index

        def __exit__(self, *_):
            at[0] = self.before

    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: at[0], raising=False)
    return at


@pytest.mark.parametrize("name", CALLS)
def test_tensors_of_another_device_are_refused(library, current, name):
    """The host's too: an address of another device's memory must not reach a kernel."""
    make, call = CALLS[name]
    takes_plan = name in ("rotary", "norm", "gradient")

    def arguments(index):
        return dict(make(index), plan=Plan(index)) if takes_plan else make(index)

    for index in (0, 1):                   # all together on either: taken
        call(arguments(index), index)
    taken = len(library.calls)
    assert taken >= 2
    for other in (-1, 1):
        for moved in arguments(0):
            with pytest.raises(ValueError):
                call(dict(arguments(0), **{moved: arguments(other)[moved]}), 0)
        if not takes_plan:
            with pytest.raises(ValueError):
                call(arguments(0), 1)      # the cache
    with pytest.raises(ValueError):
        call(arguments(-1), 0)
    assert len(library.calls) == taken


def test_plans_and_caches_are_made_on_the_current_device(monkeypatch):
    """A rank's own, not the first one's."""
    made = []
    monkeypatch.setattr(torch.Tensor, "to", lambda x, device: made.append(device) or x)
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, real=torch.empty, **more: made.append(device) or real(*a, **more))
    monkeypatch.setattr(A.KVCache, "__init__", lambda self, *a, **more: None)
    A.Rotary(64)
    A.KVCache.empty(2, 1, 64, 128, 8)
    assert [d for d in made if d is not None] == ["cuda"] * 5


def test_capture_is_asked_of_the_cache_s_device(library, current, monkeypatch):
    """While the other device's stream is captured, a workspace is kept; while its own is, none of those kept is handed over."""
    for capturing, kept in ((0, True), (1, False)):
        monkeypatch.setattr(torch._C, "_cuda_isCurrentStreamCapturing", lambda c=capturing: current[0] == c)
        library.calls.clear()
        held = []
        for _ in range(2):
            A.tree_attention(Fake(3, 4, 64, index=1), cache_of(1), *batch_of(1))
            held.append(torch.empty(4096, dtype=torch.uint8))       # what a workspace given back would be
        assert (len(A._kept.rooms) > 0) and ((library.calls[0][2] == library.calls[1][2]) or not kept)
        assert any(at == room[1] for _, _, at in library.calls for room in A._kept.rooms.values()) == kept


# ------------------------------------------------------------------------------------------------ gradients

@pytest.mark.parametrize("name,of", [("rotary", "q"), ("rotary", "k"), ("norm", "q"), ("norm", "k"), ("norm", "q_weight"), ("norm", "k_weight"), ("append", "k"),
                                     ("append", "v"), ("attention", "q")])
def test_what_requires_gradients_is_refused(library, current, name, of):
    """A result without one would end the graph silently.  Without gradients enabled there is nothing to lose."""
    make, call = CALLS[name]

    def arguments():
        a = make(0)
        a[of].requires_grad = True
        return dict(a, plan=Plan(0)) if name in ("rotary", "norm") else a

    with pytest.raises(ValueError, match="no_grad"):
        call(arguments(), 0)
    assert not library.calls
    with torch.no_grad():
        call(arguments(), 0)
    assert library.calls


def test_gradients_of_what_requires_them(library, current):
    """The backward call itself takes any tensors."""
    make, call = CALLS["gradient"]
    a = make(0)
    for x in a.values():
        x.requires_grad = True
    call(dict(a, plan=Plan(0)), 0)
    assert library.calls


# ------------------------------------------------------------------------------------------------ contexts

def test_a_table_wider_than_contexts_are_counted(library, current, monkeypatch):
    """The default context is what the table holds, up to what a call takes."""
    contexts = []
    take = library.conqur_tree_attention
    monkeypatch.setattr(library, "conqur_tree_attention", lambda call, stream: contexts.append(struct.unpack_from("=Q", call, WORKSPACE - 8)[0]) or take(call, stream),
                        raising=False)
    start, prefix, _ = batch_of()
    for columns in (4, 1 << 26):
        table = Fake(1, 1, dtype=torch.int32)
        table.host = Wide(columns)
        A.tree_attention(Fake(3, 4, 64), cache_of(), start, prefix, table)
    assert set(contexts) == {4 * 32, (1 << 31) - 1}


class Wide:
    """A table's shape without its memory."""

    def __init__(self, columns):
        self.shape, self.dtype = (1, columns), torch.int32

    def stride(self):
        return self.shape[1], 1

    def dim(self):
        return 2

    def data_ptr(self):
        return 0x1000
