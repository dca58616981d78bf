"""The attention layer around the calibrated heads, over libconqur.so (the C ABI declared in include/conqur.h).

Argument marshalling only, like `binding`: every step runs in the library's HIP kernels, PyTorch supplies device memory and
the stream (the current one of the tensors' device).  Nothing synchronises, nothing falls back to the CPU.

  Rotary                              the plan of a rotary position encoding (frequencies on the device)
  rotary                              positions into queries and keys, or back out of their gradients
  qk_norm_rotary, .._backward         per-head norms and positions in one pass, and that pass's gradients
  KVCache, append                     a paged cache of keys and values in bf16 or in 8- or 4-bit zero-point codes
  Pages                               which of its pages are taken, and by how many sequences (on the host)
  gather                              tokens of a cache into other pages: forks, tokens that are kept, beams
  tree_attention                      attention of new tokens (a tree of drafted ones, a chain, a single one) over the cache
  chunk_attention                     attention of any number of new tokens over the cache, with windows, bounds, capped scores, a bias by distance
  attention, attention_backward       attention of packed sequences over themselves, and its gradients

Rows are [tokens, heads, width] tensors of any token and head stride, e.g. slices of a fused projection's output.  All tensors of a call, its
plan and its cache lie on one device.  Nothing here is recorded for autograd: tensors that require gradients are refused where gradients are
enabled.
"""
from __future__ import annotations

import ctypes
import struct
import threading
from typing import Optional, Tuple

import torch
from torch import _C, bfloat16, contiguous_format, empty_like, float32, int32, int64

from . import binding

SCALINGS = {"none": 0, "linear": 1, "base": 2, "bands": 3, "ramp": 4}

MOST_CONTEXT = (1 << 31) - 1       # tokens of a sequence that a call counts

# The HOST structs of the header, field by field (conqur_heads: pointer, two strides, heads).
_HEADS = "QqqQ"
_ROTARY = struct.Struct("=" + 6 * _HEADS + "QQQQ" + "Q" + "IIIII" + "ff" + "I")
_CACHE_BATCH = "QQQQQIIII" + "QQQqII"
_APPEND = struct.Struct("=" + _CACHE_BATCH + 4 * _HEADS + "Q")
_TREE = struct.Struct("=" + _CACHE_BATCH + 2 * _HEADS + "QQQQQ" + "If")
_GATHER = struct.Struct("=QQQQQIIII" + "QQQQ" + "qq" + "Q" + "IIII")
_CHUNK = struct.Struct("=" + _CACHE_BATCH + 2 * _HEADS + "QQQQQQQ" + "II" + "ff" + "II")
_ATTENTION = struct.Struct("=" + 8 * _HEADS + "QQQQQ" + "Q" + "III" + "ff" + "I" + "QQ")
_ABSENT = (0, 0, 0, 0)
_NOTHING = (None, 0, 0)


def _check(status: int, what: str) -> None:
    if status != binding.OK:
        raise binding.ConqurError(status, f"{what} failed")


# A decode step makes three of these calls a layer, so what Python does around each counts as much as a small kernel: tensors are looked at with
# as few attribute reads as the checks need, torch's names are taken once, and the stream is asked for by device index (a pass of `rotary`
# 15.1 -> 10 us, of which the launch is 3.7).

def _rows(x, name: str, dtype, device: int, shape) -> Tuple[int, int, int, int]:
    stride = x.stride()
    if x.shape != shape or len(shape) != 3 or stride[2] != 1 or x.dtype is not dtype:
        raise ValueError(f"{name} must be a {list(shape)} device tensor of {dtype} with unit stride along the width")
    if x.get_device() != device:
        _elsewhere(x, name, device)
    return x.data_ptr(), stride[0], stride[1], shape[1]


def _vector(x, name: str, dtype, device: int, n: int) -> int:
    if x.dtype is not dtype or x.shape != (n,) or not x.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} device tensor of {n} entries")
    if x.get_device() != device:
        _elsewhere(x, name, device)
    return x.data_ptr()


def _elsewhere(x, name: str, device: int):
    """A kernel takes addresses as they are: what lies on the host or on another GPU must not get that far."""
    raise ValueError(f"{name} lies on {x.device}, where a tensor on " + ("a GPU" if device < 0 else f"cuda:{device}") + " is needed")


def _no_gradient(what: str, instead: str) -> None:
    """These calls are not part of autograd's graph: a result would end it without a word."""
    raise ValueError(f"{what} records nothing for autograd: {instead}; call it under torch.no_grad() or on detached tensors")


def _run(call, device: int, *args) -> int:
    """A library call's status, on a device and its current stream."""
    if device == _C._cuda_getDevice():
        return call(*args, _C._cuda_getCurrentRawStream(device))
    with torch.cuda.device(device):
        return call(*args, _C._cuda_getCurrentRawStream(device))


def _like(x):
    return None if x is None else empty_like(x, memory_format=contiguous_format)


class Rotary:
    """Frequencies of a rotary position encoding over the first `part` entries of a head.  interleaved: pairs (2j, 2j + 1) instead of
    (j, j + part/2).  scaling: "none", "linear", "base", "bands" or "ramp", for contexts `factor` times the trained `context`
    (conqur_rotary_scaling in the header says what `low` and `high` are)."""

    def __init__(self, part: int, theta: float = 10000.0, interleaved: bool = False, scaling: str = "none", factor: float = 1.0, low: float = 1.0,
                 high: float = 4.0, context: float = 8192.0, device: str = "cuda"):
        if scaling not in SCALINGS:
            raise ValueError(f"scaling must be one of {sorted(SCALINGS)}")
        turns = torch.empty(max(part // 2, 1), dtype=torch.float64)
        magnitude = ctypes.c_float()
        _check(binding.load().conqur_rotary_frequencies(part, SCALINGS[scaling], theta, factor, low, high, context, turns.data_ptr(),
                                                        ctypes.byref(magnitude)), "conqur_rotary_frequencies")
        self.part, self.layout, self.magnitude = part, 1 if interleaved else 0, magnitude.value
        self.turns = turns.to(device)


def _rotary_call(plan, q, k, positions, q_out, k_out, q_grad=None, k_grad=None, q_weight=None, k_weight=None, transposed=0, eps=0.0) -> bytes:
    dtype = q.dtype
    if dtype is not bfloat16 and dtype is not float32:
        raise ValueError("queries and keys must be bf16 or fp32")
    shape, k_shape = q.shape, None if k is None else k.shape
    if len(shape) != 3 or (k is not None and (len(k_shape) != 3 or k_shape[0] != shape[0] or k_shape[2] != shape[2])):
        raise ValueError("queries and keys must be [tokens, heads, width], with as many tokens and as wide")
    tokens, _, width = shape
    device = q.get_device()
    if device < 0:
        _elsewhere(q, "q", device)
    if plan.turns.get_device() != device:
        _elsewhere(plan.turns, "the plan", device)
    same, k_same = (dtype, device, shape), (dtype, device, k_shape)
    return _ROTARY.pack(*_rows(q, "q", *same), *(_ABSENT if k is None else _rows(k, "k", *k_same)),
                        *_rows(q_out, "the result of q", *same), *(_ABSENT if k is None else _rows(k_out, "the result of k", *k_same)),
                        *(_ABSENT if q_grad is None else _rows(q_grad, "the gradient of q", *same)),
                        *(_ABSENT if k_grad is None else _rows(k_grad, "the gradient of k", *k_same)),
                        0 if q_weight is None else _vector(q_weight, "q_weight", dtype, device, width),
                        0 if k_weight is None else _vector(k_weight, "k_weight", dtype, device, width),
                        _vector(positions, "positions", int64, device, tokens), plan.turns.data_ptr(), tokens, width, plan.part, plan.layout,
                        1 if dtype is bfloat16 else 0, transposed, plan.magnitude, eps, 0)


def rotary(plan: Rotary, q, positions, k=None, out=None, k_out=None, transposed: bool = False):
    """Queries (and keys) rotated by their positions (int64, one per token), into new tensors unless `out` / `k_out` are given (they may
    be the inputs).  transposed: the transposed rotation, for gradients.  Returns the result of q, or of (q, k)."""
    if (q.requires_grad or (k is not None and k.requires_grad)) and torch.is_grad_enabled():
        _no_gradient("rotary", "transposed=True takes gradients back")
    if out is None:
        out = _like(q)
    if k_out is None and k is not None:
        k_out = _like(k)
    call = _rotary_call(plan, q, k, positions, out, k_out, transposed=1 if transposed else 0)
    _check(_run(binding.load().conqur_rotary, q.get_device(), call), "conqur_rotary")
    return out if k is None else (out, k_out)


def qk_norm_rotary(plan: Rotary, q, k, q_weight, k_weight, positions, eps: float = 1e-6, out=None, k_out=None):
    """rotary(w x / sqrt(mean x^2 + eps)) of queries and keys, in one pass; returns (q, k)."""
    if (q.requires_grad or k.requires_grad or q_weight.requires_grad or k_weight.requires_grad) and torch.is_grad_enabled():
        _no_gradient("qk_norm_rotary", "qk_norm_rotary_backward gives its gradients")
    if out is None:
        out = _like(q)
    if k_out is None:
        k_out = _like(k)
    call = _rotary_call(plan, q, k, positions, out, k_out, q_weight=q_weight, k_weight=k_weight, eps=eps)
    _check(_run(binding.load().conqur_qk_norm_rotary, q.get_device(), call), "conqur_qk_norm_rotary")
    return out, k_out


def qk_norm_rotary_backward(plan: Rotary, q, k, q_weight, k_weight, positions, q_grad, k_grad, eps: float = 1e-6):
    """Gradients of qk_norm_rotary at inputs q, k, for the gradients q_grad, k_grad of its results: (of q, of k, of q_weight, of k_weight), the
    last two in fp32."""
    lib = binding.load()
    dq, dk = _like(q), _like(k)
    call = _rotary_call(plan, q, k, positions, dq, dk, q_grad, k_grad, q_weight, k_weight, eps=eps)
    width = q.shape[2]
    dw = torch.empty((2, width), dtype=float32, device=q.device)
    size = lib.conqur_qk_norm_rotary_workspace(width)
    workspace = torch.empty(size, dtype=torch.uint8, device=q.device)
    at = dw.data_ptr()
    _check(_run(lib.conqur_qk_norm_rotary_backward, q.get_device(), call, at, at + 4 * width, workspace.data_ptr(), size),
           "conqur_qk_norm_rotary_backward")
    return dq, dk, dw[0], dw[1]


class KVCache:
    """A pool of pages.  bits 16: k [pages, heads, page_tokens, width] and v [pages, heads, width, page_tokens] in bf16; bits 8: uint8 codes in
    the same layout; bits 4: two codes a byte, width/2 bytes in place of width.  Codes have k_scale and v_scale [pages, heads, page_tokens,
    2] in fp32, (step, offset) of every token.  page_tokens: a power of two, 16 to 256; width 64 or 128.  `empty` allocates one."""

    def __init__(self, k, v, k_scale=None, v_scale=None, bits: int = 16):
        if bits not in (16, 8, 4):
            raise ValueError("bits must be 16, 8 or 4")
        dtype = bfloat16 if bits == 16 else torch.uint8
        if k.dim() != 4 or not k.is_cuda or k.dtype != dtype or not k.is_contiguous():
            raise ValueError(f"k must be a contiguous 4-D device tensor of {dtype}")
        pages, heads, page_tokens, n = k.shape
        if tuple(v.shape) != (pages, heads, n, page_tokens) or v.dtype != dtype or v.device != k.device or not v.is_contiguous():
            raise ValueError("k must be [pages, heads, page_tokens, n] and v [pages, heads, n, page_tokens], contiguous, of one type and device")
        for s in (k_scale, v_scale):
            if bits == 16:
                if s is not None:
                    raise ValueError("a bf16 cache has no scales")
            elif s is None or s.dtype != float32 or tuple(s.shape) != (pages, heads, page_tokens, 2) or s.device != k.device or not s.is_contiguous():
                raise ValueError("codes need contiguous fp32 k_scale and v_scale [pages, heads, page_tokens, 2]")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.pages, self.heads, self.page_tokens, self.bits = pages, heads, page_tokens, bits
        self.width = n * 2 if bits == 4 else n
        self.device = k.get_device()
        self._fields = (k.data_ptr(), v.data_ptr(), 0 if k_scale is None else k_scale.data_ptr(), 0 if v_scale is None else v_scale.data_ptr(),
                        pages, heads, self.width, page_tokens, bits)

    @classmethod
    def empty(cls, pages: int, heads: int, page_tokens: int, width: int, bits: int = 16, device: str = "cuda") -> "KVCache":
        n, dtype = (width // 2, torch.uint8) if bits == 4 else (width, torch.uint8 if bits == 8 else bfloat16)
        k = torch.empty((pages, heads, page_tokens, n), dtype=dtype, device=device)
        v = torch.empty((pages, heads, n, page_tokens), dtype=dtype, device=device)
        scales = [None if bits == 16 else torch.empty((pages, heads, page_tokens, 2), dtype=float32, device=device) for _ in range(2)]
        return cls(k, v, *scales, bits=bits)


def _batch(start, prefix, table, device: int) -> Tuple:
    sequences, stride = prefix.shape[0], table.stride()
    if table.dim() != 2 or table.dtype is not int32 or stride[1] != 1 or table.shape[0] != sequences:
        raise ValueError("table must be a [sequences, columns] int32 device tensor with unit column stride")
    if table.get_device() != device:
        _elsewhere(table, "table", device)
    columns = table.shape[1]
    return (_vector(start, "start", int32, device, sequences + 1), _vector(prefix, "prefix", int32, device, sequences), table.data_ptr(),
            stride[0] if sequences > 1 else max(stride[0], columns), columns, sequences)


def append(cache: KVCache, k, v, start, prefix, table, values: bool = False, k_values=None, v_values=None):
    """New keys and values (bf16) into the cache.  Sequence b's rows are [start[b], start[b + 1]) and become its tokens prefix[b] and on;
    token i lies in slot i % page_tokens of page table[b, i // page_tokens] (int32 device tensors).  A start below the one before it: no rows;
    not with more than 512 sequences, whose starts must not fall.  values (8 or 4 bits): also returns
    what the cache holds of them, (k_values, v_values), in the given or in new bf16 tensors, where rows of
    tokens without a place are not written."""
    if (k.requires_grad or v.requires_grad) and torch.is_grad_enabled():
        _no_gradient("append", "it has no gradient")
    tokens = k.shape[0]
    device = cache.device
    same = (bfloat16, device, (tokens, cache.heads, cache.width))
    if values:
        k_values = _like(k) if k_values is None else k_values
        v_values = _like(v) if v_values is None else v_values
    call = _APPEND.pack(*cache._fields, *_batch(start, prefix, table, device), *_rows(k, "k", *same), *_rows(v, "v", *same),
                        *(_ABSENT if k_values is None else _rows(k_values, "k_values", *same)),
                        *(_ABSENT if v_values is None else _rows(v_values, "v_values", *same)), tokens)
    _check(_run(binding.load().conqur_cache_append, device, call), "conqur_cache_append")
    return (k_values, v_values) if values else None


class Pages:
    """Which pages of a cache are taken, and how often, on the host: a program takes pages for new tokens, shares those that a fork has in common with
    its parent, and gives back what a sequence no longer needs.  A page is free again when every holder has given it back; the cache is not touched, and
    work that is under way on the device may still read a page that was given back: what is taken next is written behind it on the same stream."""

    def __init__(self, pages: int):
        self._free = list(range(pages - 1, -1, -1))
        self._held = [0] * pages

    @property
    def left(self) -> int:
        return len(self._free)

    def held(self, page: int) -> int:
        """By how many sequences a page is held."""
        return self._held[self._known(page)]

    def _known(self, page: int) -> int:
        if not 0 <= page < len(self._held):
            raise ValueError(f"page {page} is none of {len(self._held)}")
        return page

    def take(self, n: int) -> list:
        """n free pages, the lowest first among those never given back; none are taken if there are not enough."""
        if n < 0 or n > len(self._free):
            raise ValueError(f"{n} pages asked for, {len(self._free)} are free")
        taken = [self._free.pop() for _ in range(n)]
        for page in taken:
            self._held[page] = 1
        return taken

    def share(self, pages) -> None:
        """One more holder for each of the pages (a page named twice: two more)."""
        pages = list(pages)
        for page in pages:
            if not self._held[self._known(page)]:
                raise ValueError(f"page {page} is free")
        for page in pages:
            self._held[page] += 1

    def release(self, pages) -> list:
        """One holder fewer for each; returns the pages that are free now.  All or, with an error, none are given back."""
        pages = list(pages)
        less = {}
        for page in pages:
            less[page] = less.get(page, 0) + 1
            if less[page] > self._held[self._known(page)]:
                raise ValueError(f"page {page} is not held that often")
        freed = []
        for page in pages:
            self._held[page] -= 1
            if not self._held[page]:
                freed.append(page)
        self._free += reversed(freed)
        return freed


def gather(cache: KVCache, tokens, start, table, to_table) -> None:
    """Tokens of a cache into other pages, all heads, as they are held: tokens (int32) of sequence b, [start[b], start[b + 1]) of them (int32
    [sequences + 1], not falling), counted in its pages table[b], become tokens 0, 1, ... of the pages to_table[b] (both int32 [sequences, columns]).  A fork copies
    the page that is not full; a sequence that drops tokens names those that it keeps.  A slot that is written must not be one that the call reads, nor be
    written twice; tokens without a place in either table are not moved."""
    device = cache.device
    count, sequences = tokens.shape[0], start.shape[0] - 1
    if sequences < 1:
        raise ValueError("start must hold the sequences' first tokens and the last one's end")
    strides = []
    for x, name in ((table, "table"), (to_table, "to_table")):
        stride = x.stride()
        if x.dim() != 2 or x.dtype is not int32 or stride[1] != 1 or x.shape[0] != sequences:
            raise ValueError(f"{name} must be a [sequences, columns] int32 device tensor with unit column stride")
        if x.get_device() != device:
            _elsewhere(x, name, device)
        strides.append(stride[0] if sequences > 1 else max(stride[0], x.shape[1]))
    call = _GATHER.pack(*cache._fields, _vector(tokens, "tokens", int32, device, count), _vector(start, "start", int32, device, sequences + 1),
                        table.data_ptr(), to_table.data_ptr(), *strides, count, table.shape[1], to_table.shape[1], sequences, 0)
    _check(_run(binding.load().conqur_cache_gather, device, call), "conqur_cache_gather")


class _Kept(threading.local):
    """The workspaces of tree_attention, each thread its own, by device and stream.  A call's launches meet in it: the calls of one thread on one
    stream come one behind the other, whatever their caches, those of two threads may be enqueued between each other's launches."""

    def __init__(self):
        self.rooms = {}


_kept = _Kept()


def tree_attention(q, cache: KVCache, start, prefix, table, mask=None, max_query: int = 64, max_context: Optional[int] = None,
                   scale: Optional[float] = None, out=None):
    """Attention of new tokens q (bf16 [tokens, heads, width]; packed as in `append`, which has put their keys and values into the cache) over
    the committed tokens and those new ones that mask (int64, bit j: new token j of the sequence) names; None: each sees itself and those
    before it.  max_query: most new tokens of a sequence (up to 64); max_context: most tokens, committed and new (default: what the table
    holds; a closer bound shares the work out better).  scale: 1 / sqrt(width) unless given.  Returns out.  Rows beyond max_query of a sequence
    and rows of no sequence have no result: they stay as they are in `out`; in a new tensor, rows beyond 64 of a sequence are zeros, and all of them
    where there are more tokens than sequences of max_query hold."""
    if q.requires_grad and torch.is_grad_enabled():
        _no_gradient("tree_attention", "it has no gradient")
    if q.dim() != 3:
        raise ValueError("q must be [tokens, heads, width]")
    device = cache.device
    if _C._cuda_getDevice() != device:       # (what is asked below is asked of the current device)
        with torch.cuda.device(device):
            return tree_attention(q, cache, start, prefix, table, mask, max_query, max_context, scale, out)
    tokens, heads, _ = q.shape
    width = cache.width
    if out is None:
        out = _like(q)
        # (a max_query below 64 is the caller's word, unless the tokens are too many for it)
        if tokens > max_query and (max_query >= 64 or tokens > prefix.shape[0] * max_query):
            out.zero_()
    same = (bfloat16, device, (tokens, heads, width))
    fields = (*cache._fields, *_batch(start, prefix, table, device), *_rows(q, "q", *same), *_rows(out, "out", *same),
              0 if mask is None else _vector(mask, "mask", int64, device, tokens), tokens,
              min(table.shape[1] * cache.page_tokens, MOST_CONTEXT) if max_context is None else max_context)
    tail = (max_query, width ** -0.5 if scale is None else scale)
    lib = binding.load()
    _in_room(lib.conqur_tree_attention, lib.conqur_tree_attention_workspace, _TREE, fields, tail, q, "conqur_tree_attention")
    return out


def _in_room(call, size_of, form, fields, tail, x, what: str) -> None:
    """A call in the thread's workspace for the stream of x's device, which is the current one; its address and size stand between `fields` and `tail`."""
    device = x.get_device()
    at = device, _C._cuda_getCurrentRawStream(device)
    # (a graph keeps the room it was captured with: it takes its own, from its memory pool)
    capturing = _C._cuda_isCurrentStreamCapturing()
    rooms = _kept.rooms
    have = _NOTHING if capturing else rooms.get(at, _NOTHING)
    status = call(form.pack(*fields, *have[1:], *tail), at[1])
    if status == binding.EINVAL:       # perhaps for want of room alone: one that is large enough stays
        size = size_of(form.pack(*fields, 0, 0, *tail))
        if size > have[2]:
            room = torch.empty(size, dtype=torch.uint8, device=x.device)
            have = (room, room.data_ptr(), size)
            if not capturing:
                rooms[at] = have
            status = call(form.pack(*fields, *have[1:], *tail), at[1])
    _check(status, what)


def chunk_attention(q, cache: KVCache, start, prefix, table, first=None, last=None, window: int = 0, cap: float = 0.0, slopes=None,
                    max_query: Optional[int] = None, max_context: Optional[int] = None, scale: Optional[float] = None, out=None):
    """Attention of any number of new tokens q (bf16 [tokens, heads, width]; packed as in `append`, which has put their keys and values into the
    cache; no row two sequences') over their sequences' tokens, committed and new.  A token sees itself and those before it, or those from first on up
    to, not including, last (int32, one per row of q, counted in tokens of the sequence; first >= last: nothing, zeros); window: and at most that many, itself
    the last.  cap (up to 4096): scores become cap tanh(score / cap); slopes (fp32 [heads]): less slope times the distance.  max_query: most new tokens of
    a sequence, max_context: most tokens, committed and new (default: what q and the table hold; closer bounds choose the quicker kernel and share the work
    out better).  scale: 1 / sqrt(width) unless given.  Returns out.  Rows beyond max_query of a sequence and rows of no sequence are zeros in a new tensor and
    stay as they are in a given `out`.  Calls over long contexts need a workspace, up to 512 MiB, which the thread keeps for the stream."""
    if q.requires_grad and torch.is_grad_enabled():
        _no_gradient("chunk_attention", "it has no gradient")
    if q.dim() != 3:
        raise ValueError("q must be [tokens, heads, width]")
    device = cache.device
    if _C._cuda_getDevice() != device:
        with torch.cuda.device(device):
            return chunk_attention(q, cache, start, prefix, table, first, last, window, cap, slopes, max_query, max_context, scale, out)
    tokens, heads, _ = q.shape
    width = cache.width
    new = out is None
    if new:
        out = _like(q)
    if not 0 <= window < 1 << 31:
        raise ValueError("window must be 0 (none) or a number of tokens")
    same = (bfloat16, device, (tokens, heads, width))
    fields = (*cache._fields, *_batch(start, prefix, table, device), *_rows(q, "q", *same), *_rows(out, "out", *same),
              0 if first is None else _vector(first, "first", int32, device, tokens), 0 if last is None else _vector(last, "last", int32, device, tokens),
              0 if slopes is None else _vector(slopes, "slopes", float32, device, heads), tokens,
              min(table.shape[1] * cache.page_tokens, MOST_CONTEXT) if max_context is None else max_context)
    tail = (max(tokens, 1) if max_query is None else max_query, window, cap, width ** -0.5 if scale is None else scale, 1 if new else 0, 0)
    lib = binding.load()
    _in_room(lib.conqur_chunk_attention, lib.conqur_chunk_attention_workspace, _CHUNK, fields, tail, q, "conqur_chunk_attention")
    return out


def _attention_call(q, k, v, out, start, first, last, window: int, cap: float, slopes, scale: Optional[float], lse: int, zero_rest: bool, gradients=None) -> Tuple:
    """The call's fields but for its workspace, and its device."""
    shape, k_shape = q.shape, k.shape
    if len(shape) != 3 or len(k_shape) != 3 or k_shape[0] != shape[0] or k_shape[2] != shape[2]:
        raise ValueError("queries, keys and values must be [tokens, heads, width], with as many tokens and as wide")
    tokens, heads, width = shape
    device = q.get_device()
    if device < 0:
        _elsewhere(q, "q", device)
    if start.dim() != 1 or start.shape[0] < 2:
        raise ValueError("start must hold the sequences' first rows and the last one's end")
    same, k_same = (bfloat16, device, shape), (bfloat16, device, k_shape)
    rows = (*_rows(q, "q", *same), *_rows(k, "k", *k_same), *_rows(v, "v", *k_same), *_rows(out, "out", *same))
    if gradients is None:
        rows += 4 * _ABSENT
    else:
        grad, dq, dk, dv = gradients
        rows += (*_rows(grad, "grad", *same), *_rows(dq, "the gradient of q", *same), *_rows(dk, "the gradient of k", *k_same),
                 *_rows(dv, "the gradient of v", *k_same))
    if not 0 <= window < 1 << 31:
        raise ValueError("window must be 0 (none) or a number of tokens")
    sequences = start.shape[0] - 1
    return (*rows, lse, _vector(start, "start", int32, device, sequences + 1), 0 if first is None else _vector(first, "first", int32, device, tokens),
            0 if last is None else _vector(last, "last", int32, device, tokens), 0 if slopes is None else _vector(slopes, "slopes", float32, device, heads),
            tokens, sequences, width, window, cap, width ** -0.5 if scale is None else scale, 1 if zero_rest else 0), device


def _with_room(call, size_of, fields, x, device: int, without: bool) -> int:
    """A call's status, with the workspace that it asks for, if any; without: most such calls need none, and only one that is refused is asked."""
    alone = _ATTENTION.pack(*fields, 0, 0)
    if without:
        status = _run(call, device, alone)
        if status != binding.EINVAL:
            return status
    size = size_of(alone)
    if not size:
        return binding.EINVAL if without else _run(call, device, alone)
    room = torch.empty(size, dtype=torch.uint8, device=x.device)
    return _run(call, device, _ATTENTION.pack(*fields, room.data_ptr(), size))


def attention(q, k, v, start, first=None, last=None, window: int = 0, cap: float = 0.0, slopes=None, scale: Optional[float] = None, lse: bool = False,
              out=None):
    """Attention of packed sequences over themselves: q [tokens, heads, width], k and v [tokens, key heads, width], bf16, heads a multiple of the key
    heads (up to 64 times); start (int32 [sequences + 1], not falling): sequence b's tokens are the rows [start[b], start[b + 1]).  width: 32, 64, 80, 96
    or 128.  A token sees itself and those before it, or, of its sequence's tokens, those from first on up to, not including, last (int32, one per
    row of q): documents in a sequence, prefixes seen from both sides, padding that sees nothing (first >= last: zeros); window: and at most that many, itself the
    last.  cap (up to 4096): scores become cap tanh(score / cap); slopes (fp32 [heads]): less slope times the distance.  scale: 1 / sqrt(width) unless given.
    Returns out, or (out, lse): fp32 [tokens, heads], the logarithms of the rows' sums.  Rows of no sequence are zeros in a new tensor (lse -inf)
    and stay as they are in a given `out` (their lse is then not written)."""
    if (q.requires_grad or k.requires_grad or v.requires_grad) and torch.is_grad_enabled():
        _no_gradient("attention", "attention_backward gives its gradients")
    new = out is None
    if new:
        out = _like(q)
    sums = torch.empty((q.shape[0], q.shape[1]), dtype=float32, device=q.device) if lse else None
    fields, device = _attention_call(q, k, v, out, start, first, last, window, cap, slopes, scale, 0 if sums is None else sums.data_ptr(), new)
    lib = binding.load()
    _check(_with_room(lib.conqur_attention, lib.conqur_attention_workspace, fields, q, device, True), "conqur_attention")
    return (out, sums) if lse else out


def attention_backward(q, k, v, out, lse, grad, start, first=None, last=None, window: int = 0, cap: float = 0.0, slopes=None,
                       scale: Optional[float] = None):
    """Gradients of attention (of q, of k, of v) for the gradient `grad` of its result `out` (bf16), with the lse that it gave and the other arguments as
    it took them.  Rows of no sequence get zeros.  What is not finite in a row's query or gradient, or in a key or value that it sees, may make NaN of the
    gradients of that row and of all that it sees, also where its result is finite; of no others."""
    if lse.dtype is not float32 or q.dim() != 3 or lse.shape != (q.shape[0], q.shape[1]) or not lse.is_contiguous():
        raise ValueError("lse must be a contiguous fp32 device tensor [tokens, heads]")
    if lse.get_device() != q.get_device():
        _elsewhere(lse, "lse", q.get_device())
    gradients = grad, _like(q), _like(k), _like(v)
    fields, device = _attention_call(q, k, v, out, start, first, last, window, cap, slopes, scale, lse.data_ptr(), True, gradients)
    lib = binding.load()
    _check(_with_room(lib.conqur_attention_backward, lib.conqur_attention_backward_workspace, fields, q, device, False), "conqur_attention_backward")
    return gradients[1:]
